// pages.cu -- the pages and rows of the KV cache: reserve, release, fork (page
// bookkeeping on the device), append and prune (row movement).
//
// Bookkeeping works on a page table [B, P] and a count of holders per page; a
// page is free when its count is 0, and free pages are handed out lowest id
// first, so results do not depend on scheduling (the only atomics are integer
// adds and minima). Row movement is bound by HBM: every moved byte is read and
// written once, in 16-byte columns.
#include <limits.h>

#include <algorithm>

#include "common.cuh"

namespace dreams {
namespace {

constexpr int PAGE = 64;
constexpr int BOOK_THREADS = 1024;
constexpr int FORK_CTAS = 8;  // one portable cluster

struct Pool {
  int32_t *table;
  int32_t *ref;
  int32_t B, P, num_pages;
};

struct Cache {
  uint4 *k, *v;  // 16-byte columns
  int32_t n_layers;
  int64_t layer16;  // layer stride in 16-byte units
  int32_t row16;    // Hkv * D / 8: 16-byte columns of a slot
  int32_t capacity;
  const int32_t *table;  // nullptr: contiguous
  int32_t P, num_pages;
};

// 16-byte offset of slot s of sequence b within a layer; -1: no page.
__device__ __forceinline__ int64_t slot16(const Cache &c, int b, int s) {
  if (c.table == nullptr) return (int64_t(b) * c.capacity + s) * c.row16;
  const int pg = __ldg(c.table + int64_t(b) * c.P + (s >> 6));
  if (pg < 0 || pg >= c.num_pages) return -1;
  return (int64_t(pg) * PAGE + (s & (PAGE - 1))) * c.row16;
}

__device__ __forceinline__ uint4 ld_stream(const uint4 *p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p)
               : "memory");
  return v;
}

// Exclusive prefix sum of one value per thread over the block, and the total.
__device__ __forceinline__ int block_scan(int x, int *s_warp, int &total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int y = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int z = __shfl_up_sync(0xffffffffu, y, o);
    if (lane >= o) y += z;
  }
  __syncthreads();  // the last use of s_warp is over
  if (lane == 31) s_warp[warp] = y;
  __syncthreads();
  int w = lane < int(blockDim.x >> 5) ? s_warp[lane] : 0;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int z = __shfl_up_sync(0xffffffffu, w, o);
    if (lane >= o) w += z;
  }
  total = __shfl_sync(0xffffffffu, w, 31);
  const int before = __shfl_sync(0xffffffffu, w, warp > 0 ? warp - 1 : 0);
  return y - x + (warp > 0 ? before : 0);
}

// Writes the free pages among [lo, hi), lowest first, to list[0 .. most); returns
// how many there are, counting no further than `most`. (One block.)
__device__ int list_free(const int32_t *ref, int lo, int hi, int most, int32_t *list, int *s_warp) {
  int found = 0;
  for (int base = lo; base < hi && found < most; base += 4 * int(blockDim.x)) {
    const int at = base + 4 * int(threadIdx.x);
    int f[4], n = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[i] = at + i < hi && __ldcg(ref + at + i) == 0;
      n += f[i];
    }
    int total;
    int r = found + block_scan(n, s_warp, total);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (f[i]) {
        if (r < most) list[r] = at + i;
        ++r;
      }
    found += total;
  }
  return ::min(found, most);
}

// ------------------------------------------------------------------ reserve
// One block: rows in chunks of its threads, each thread counting what its row
// lacks; a prefix sum gives every row its place in the list of free pages. A
// call is a few microseconds of dependent loads, whatever the pool's size up
// to about 10^5 pages.
__global__ void __launch_bounds__(BOOK_THREADS) kv_reserve_kernel(const Pool p, const int32_t *kv_len,
                                                                  const int32_t *n_new, int32_t *start,
                                                                  int32_t *list, int32_t *status) {
  __shared__ int s_warp[32];
  const int64_t cap = int64_t(p.P) * PAGE;
  int base = 0;
  for (int b0 = 0; b0 < p.B; b0 += BOOK_THREADS) {
    const int b = b0 + int(threadIdx.x);
    int need = 0;
    if (b < p.B) {
      const int64_t L = __ldg(kv_len + b), n = __ldg(n_new + b);
      if (L < 0 || n < 0 || L + n > cap) {
        flag(status, DREAMS_DATA_BAD_KV_LEN);
      } else if (n > 0) {
        const int e1 = int((L + n + PAGE - 1) / PAGE);
        int bad = 0;
        for (int e = int(L / PAGE); e < e1; ++e) {
          const int pg = p.table[int64_t(b) * p.P + e];
          if (pg == -1) ++need;
          else if (pg < 0 || pg >= p.num_pages) bad |= DREAMS_DATA_BAD_PAGE;
          else if (__ldcg(p.ref + pg) != 1) bad |= DREAMS_DATA_SHARED_PAGE;
        }
        if (bad) {
          flag(status, bad);
          need = 0;
        }
      }
    }
    int total;
    const int r = base + block_scan(need, s_warp, total);
    if (b < p.B) start[b] = need > 0 ? r : -1;
    base += total;
  }
  if (base == 0) return;
  const int have = list_free(p.ref, 0, p.num_pages, ::min(base, p.num_pages), list, s_warp);
  __syncthreads();  // start[] and list[] are written
  for (int b = int(threadIdx.x); b < p.B; b += BOOK_THREADS) {
    int r = start[b];
    if (r < 0) continue;
    const int L = __ldg(kv_len + b);
    const int e0 = L / PAGE, e1 = int((int64_t(L) + __ldg(n_new + b) + PAGE - 1) / PAGE);
    int32_t *row = p.table + int64_t(b) * p.P;
    int need = 0;
    for (int e = e0; e < e1; ++e) need += row[e] == -1;
    if (r + need > have) {
      flag(status, DREAMS_DATA_NO_PAGES);
      continue;
    }
    for (int e = e0; e < e1; ++e)
      if (row[e] == -1) {
        const int pg = list[r++];
        row[e] = pg;
        p.ref[pg] = 1;
      }
  }
}

// ------------------------------------------------------------------ release
// One thread per table entry.
__global__ void __launch_bounds__(256) kv_release_kernel(const Pool p, const int32_t *begin, const int32_t *end,
                                                         int32_t *status) {
  const int b = blockIdx.y;
  const int e = blockIdx.x * 256 + threadIdx.x;
  const int64_t lo = __ldg(begin + b), hi = __ldg(end + b);
  if (lo < 0 || hi > int64_t(p.P) * PAGE) {
    if (e == 0) flag(status, DREAMS_DATA_BAD_KV_LEN);
    return;
  }
  if (e >= p.P || int64_t(e) * PAGE < lo || int64_t(e + 1) * PAGE > hi) return;
  int32_t *at = p.table + int64_t(b) * p.P + e;
  const int pg = *at;
  if (pg == -1) return;
  if (pg < 0 || pg >= p.num_pages) {
    flag(status, DREAMS_DATA_BAD_PAGE);
    return;
  }
  atomicSub(p.ref + pg, 1);
  *at = -1;
}

// ------------------------------------------------------------------ fork
// What the two launches share, in the workspace.
struct ForkState {
  int32_t *head;   // [0] data flags, [1] copies, [2 + c] free pages found by CTA c
  int32_t *first;  // [B] the lowest row of each parent (B: none)
  int32_t *len;    // [B] new lengths
  int32_t *src, *dst, *rows;  // [B] copies: page, new page, rows of it
  int32_t *list;   // [FORK_CTAS][B] free pages by CTA
  int32_t *table;  // [B, P] the new table
};
constexpr int FORK_HEAD = 2 + FORK_CTAS;

// (Not the .aligned forms: warps come here from loops that their lanes left at
// different turns.)
__device__ __forceinline__ void cluster_sync() {
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release;\n barrier.cluster.wait.acquire;" ::: "memory");
}

// The new table, counts and lengths, and the list of pages to copy: one
// cluster, whose barrier separates the phases (new entries from the old table;
// counts; free pages; the table).
__global__ void __cluster_dims__(FORK_CTAS, 1, 1) __launch_bounds__(BOOK_THREADS)
    kv_fork_table_kernel(const Pool p, const int32_t *parent, const int32_t *kv_len, int32_t *new_kv_len,
                         const ForkState f, int32_t *status) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  __shared__ int s_warp[32];
  const int rank = blockIdx.x;
  const int t0 = rank * BOOK_THREADS + int(threadIdx.x), nt = FORK_CTAS * BOOK_THREADS;
  const int64_t cells = int64_t(p.B) * p.P;
  const int64_t cap = int64_t(p.P) * PAGE;

  if (t0 < FORK_HEAD) f.head[t0] = 0;
  for (int b = t0; b < p.B; b += nt) f.first[b] = p.B;
  cluster_sync();
  for (int i = t0; i < p.B; i += nt) {
    const int q = __ldg(parent + i);
    if (q < -1 || q >= p.B) {
      atomicOr(f.head, DREAMS_DATA_BAD_INDEX);
      f.len[i] = 0;
      continue;
    }
    const int L = q < 0 ? 0 : __ldcg(kv_len + q);
    if (L < 0 || L > cap) atomicOr(f.head, DREAMS_DATA_BAD_KV_LEN);
    if (q >= 0) atomicMin(f.first + q, i);
    f.len[i] = L;
  }
  cluster_sync();
  if (__ldcg(f.head) == 0) {
    for (int64_t x = t0; x < cells; x += nt) {
      const int i = int(x / p.P), e = int(x - int64_t(i) * p.P);
      const int q = __ldg(parent + i);
      const int old = __ldcg(p.table + x);
      int bad = old < -1 || old >= p.num_pages;
      int now = -1;
      if (q >= 0) {
        const int src = __ldcg(p.table + int64_t(q) * p.P + e);
        const int L = __ldcg(f.len + i), full = L / PAGE;
        const bool keeps = __ldcg(f.first + q) == i;
        const bool part = e == full && L % PAGE != 0;
        bad |= part && src < 0;
        now = keeps || e < full ? src : -1;
      }
      if (bad) atomicOr(f.head, DREAMS_DATA_BAD_PAGE);
      f.table[x] = now;
    }
  }
  cluster_sync();
  bool ok = __ldcg(f.head) == 0;
  if (ok) {
    for (int64_t x = t0; x < cells; x += nt) {
      const int old = __ldcg(p.table + x), now = f.table[x];
      if (old == now) continue;
      if (old >= 0) atomicSub(p.ref + old, 1);
      if (now >= 0) atomicAdd(p.ref + now, 1);
    }
  }
  cluster_sync();
  // the free pages of each CTA's part of the pool, at most B of them
  const int part = (p.num_pages + FORK_CTAS - 1) / FORK_CTAS;
  if (ok) {
    const int lo = ::min(p.num_pages, rank * part);
    const int found = list_free(p.ref, lo, ::min(p.num_pages, lo + part), p.B, f.list + int64_t(rank) * p.B, s_warp);
    if (threadIdx.x == 0) f.head[2 + rank] = found;
  }
  cluster_sync();
  // rows that get a copy of their parent's last page, in order (CTA 0)
  if (ok && rank == 0) {
    int have[FORK_CTAS], all = 0;
#pragma unroll
    for (int c = 0; c < FORK_CTAS; ++c) {
      have[c] = __ldcg(f.head + 2 + c);
      all += have[c];
    }
    int base = 0;
    for (int i0 = 0; i0 < p.B; i0 += BOOK_THREADS) {
      const int i = i0 + int(threadIdx.x);
      int need = 0, q = -1, L = 0;
      if (i < p.B) {
        q = __ldg(parent + i);
        L = __ldcg(f.len + i);
        need = q >= 0 && __ldcg(f.first + q) != i && L % PAGE != 0;
      }
      int total;
      const int r = base + block_scan(need, s_warp, total);
      if (need && r < all) {
        int c = 0, at = r;
        while (at >= have[c]) at -= have[c++];
        f.src[r] = __ldcg(p.table + int64_t(q) * p.P + L / PAGE);
        f.dst[r] = __ldcg(f.list + int64_t(c) * p.B + at);
        f.rows[r] = L % PAGE;
        f.table[int64_t(i) * p.P + L / PAGE] = f.dst[r];
      }
      base += total;
    }
    if (base > all) {
      if (threadIdx.x == 0) f.head[0] = DREAMS_DATA_NO_PAGES;
    } else {
      __syncthreads();
      for (int r = int(threadIdx.x); r < base; r += BOOK_THREADS) p.ref[f.dst[r]] = 1;
      if (threadIdx.x == 0) f.head[1] = base;
    }
  }
  cluster_sync();
  const int bad = __ldcg(f.head);
  if (bad) {
    // nothing changes: the counts go back
    if (ok)
      for (int64_t x = t0; x < cells; x += nt) {
        const int old = __ldcg(p.table + x);
        int now = __ldcg(f.table + x);
        // an entry filled in for a copy was not counted
        const int i = int(x / p.P), q = __ldg(parent + i);
        if (q >= 0 && __ldcg(f.first + q) != i && int(x - int64_t(i) * p.P) == __ldcg(f.len + i) / PAGE) now = -1;
        if (old == now) continue;
        if (old >= 0) atomicAdd(p.ref + old, 1);
        if (now >= 0) atomicSub(p.ref + now, 1);
      }
    if (t0 == 0) flag(status, bad);
    if (new_kv_len != kv_len)
      for (int i = t0; i < p.B; i += nt) new_kv_len[i] = __ldcg(kv_len + i);
    return;
  }
  for (int64_t x = t0; x < cells; x += nt) {
    const int now = __ldcg(f.table + x);
    if (__ldcg(p.table + x) != now) p.table[x] = now;
  }
  for (int i = t0; i < p.B; i += nt) new_kv_len[i] = __ldcg(f.len + i);
}

// The copies, in pieces of 256 threads x 4 x 16 bytes. A page is contiguous
// within a layer, so its first `rows` rows are one run of 16-byte columns.
constexpr int COPY_PIECE = 1024;
__global__ void __launch_bounds__(256) kv_fork_copy_kernel(const Cache c, const ForkState f, int pieces) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int n = __ldcg(f.head + 1);
  const int64_t items = int64_t(n) * c.n_layers * 2 * pieces;
  for (int64_t x = blockIdx.x; x < items; x += gridDim.x) {
    const int piece = int(x % pieces);
    int64_t y = x / pieces;
    uint4 *base = (y & 1) ? c.v : c.k;
    y >>= 1;
    const int layer = int(y % c.n_layers), r = int(y / c.n_layers);
    const int len = __ldcg(f.rows + r) * c.row16;
    base += layer * c.layer16;
    const uint4 *src = base + int64_t(__ldcg(f.src + r)) * PAGE * c.row16;
    uint4 *dst = base + int64_t(__ldcg(f.dst + r)) * PAGE * c.row16;
    const int at = piece * COPY_PIECE + int(threadIdx.x);
    uint4 v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (at + 256 * i < len) v[i] = ld_stream(src + at + 256 * i);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (at + 256 * i < len) dst[at + 256 * i] = v[i];
  }
}

// ------------------------------------------------------------------ append
// Units are 16-byte columns of (sequence, token); each thread moves K and V of
// up to four.
constexpr int APPEND_UNROLL = 4;
__global__ void __launch_bounds__(256) kv_append_kernel(const Cache c, const uint4 *k_new, const uint4 *v_new,
                                                        int64_t sb16, int64_t st16, const int32_t *kv_len,
                                                        const int32_t *n_new, int T_max, int32_t *status) {
  const int b = blockIdx.y;
  const int n = __ldg(n_new + b);
  const int64_t L = __ldg(kv_len + b);
  if (n < 0 || n > T_max || L < 0 || L + n > c.capacity) {
    if (blockIdx.x == 0 && threadIdx.x == 0) flag(status, DREAMS_DATA_BAD_KV_LEN);
    return;
  }
  const int64_t units = int64_t(n) * c.row16;
  const int64_t u0 = int64_t(blockIdx.x) * (256 * APPEND_UNROLL) + threadIdx.x;
  uint4 kk[APPEND_UNROLL], vv[APPEND_UNROLL];
  int64_t to[APPEND_UNROLL];
#pragma unroll
  for (int i = 0; i < APPEND_UNROLL; ++i) {
    const int64_t u = u0 + 256 * i;
    to[i] = -1;
    if (u < units) {
      const int t = int(u / c.row16), col = int(u - int64_t(t) * c.row16);
      const int64_t from = b * sb16 + t * st16 + col;
      kk[i] = ld_stream(k_new + from);
      vv[i] = ld_stream(v_new + from);
      const int64_t s = slot16(c, b, int(L) + t);
      if (s < 0) flag(status, DREAMS_DATA_BAD_PAGE);
      else to[i] = s + col;
    }
  }
#pragma unroll
  for (int i = 0; i < APPEND_UNROLL; ++i)
    if (to[i] >= 0) {
      c.k[to[i]] = kk[i];
      c.v[to[i]] = vv[i];
    }
}

// ------------------------------------------------------------------ prune
// A slot moves down (or stays), and a later slot never lands above an earlier
// one's source: walking a sequence upwards, the rows of a step can be written
// once they have been read, and no later step's source is written before it is
// read. A CTA walks one column block of (layer, K or V, sequence); column
// blocks are independent. CW16: 16-byte columns of a block.
constexpr int PRUNE_THREADS = 256, PRUNE_UNROLL = 4;
template <int CW16>
__global__ void __launch_bounds__(PRUNE_THREADS) kv_prune_kernel(const Cache c, const int32_t *keep, int v0, int n_vis,
                                                                 int r, const int32_t *kv_len, const int32_t *ref,
                                                                 int32_t *new_kv_len, int32_t *status) {
  constexpr int RPS = PRUNE_THREADS / CW16;  // rows read at a time
  constexpr int STEP = RPS * PRUNE_UNROLL;
  const int b = blockIdx.y;
  const int nblk = (c.row16 + CW16 - 1) / CW16;
  const int blk = blockIdx.x % nblk, rest = blockIdx.x / nblk;
  const bool reporter = blockIdx.x == 0 && threadIdx.x == 0;
  const int L = __ldg(kv_len + b);
  const int32_t *list = keep + int64_t(b) * r;
  __shared__ int s_bad;
  if (threadIdx.x == 0) s_bad = 0;
  __syncthreads();
  int bad = 0;
  if (L > c.capacity || int64_t(v0) + n_vis > L) {
    bad = DREAMS_DATA_BAD_KV_LEN;
  } else {
    for (int i = threadIdx.x; i < r; i += PRUNE_THREADS) {
      const int s = __ldg(list + i), before = i ? __ldg(list + i - 1) : v0 - 1;
      if (s <= before || s >= v0 + n_vis) bad |= DREAMS_DATA_BAD_INDEX;
    }
    if (c.table != nullptr)
      for (int e = v0 / PAGE + int(threadIdx.x); e * PAGE < L; e += PRUNE_THREADS) {
        const int pg = __ldg(c.table + int64_t(b) * c.P + e);
        if (pg < 0 || pg >= c.num_pages) bad |= DREAMS_DATA_BAD_PAGE;
        else if (ref != nullptr && __ldg(ref + pg) != 1) bad |= DREAMS_DATA_SHARED_PAGE;
      }
  }
  if (bad) atomicOr(&s_bad, bad);
  __syncthreads();
  bad = s_bad;
  if (reporter) {
    if (bad) flag(status, bad);
    new_kv_len[b] = bad ? L : L - (n_vis - r);
  }
  if (bad) return;
  const int shift = n_vis - r, n = L - v0 - shift;  // rows from v0 on afterwards
  if (shift == 0) return;
  uint4 *base = ((rest & 1) ? c.v : c.k) + int64_t(rest >> 1) * c.layer16;
  const int col = blk * CW16 + int(threadIdx.x) % CW16;
  const int tr = int(threadIdx.x) / CW16;
  const bool in = col < c.row16;
  for (int i0 = 0; i0 < n; i0 += STEP) {
    uint4 v[PRUNE_UNROLL];
    int64_t to[PRUNE_UNROLL];
#pragma unroll
    for (int j = 0; j < PRUNE_UNROLL; ++j) {
      const int i = i0 + j * RPS + tr;
      to[j] = -1;
      if (in && i < n) {
        const int s = i < r ? __ldg(list + i) : v0 + i + shift;
        if (s != v0 + i) {
          to[j] = slot16(c, b, v0 + i) + col;
          v[j] = ld_stream(base + slot16(c, b, s) + col);
        }
      }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < PRUNE_UNROLL; ++j)
      if (to[j] >= 0) base[to[j]] = v[j];
  }
}

// ------------------------------------------------------------------ host side
inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

bool cache_ok(const dreams_kv_cache_t *kv, Cache &c) {
  if (kv == nullptr || kv->k == nullptr || kv->v == nullptr || kv->n_layers < 1 || kv->Hkv < 1 || kv->D < 8 ||
      kv->D % 8 != 0 || kv->capacity < 1 || kv->layer_stride < 0)
    return false;
  if (!aligned16(kv->k) || !aligned16(kv->v) || (kv->layer_stride * 2) % 16 != 0) return false;
  if (int64_t(kv->Hkv) * (kv->D / 8) > (1 << 20)) return false;
  if (kv->page_table != nullptr &&
      (kv->page_size != PAGE || kv->pages_per_seq < 1 || kv->num_pages < 1 || !aligned4(kv->page_table) ||
       int64_t(kv->pages_per_seq) * PAGE != kv->capacity))
    return false;
  c.k = static_cast<uint4 *>(kv->k);
  c.v = static_cast<uint4 *>(kv->v);
  c.n_layers = kv->n_layers;
  c.layer16 = kv->layer_stride * 2 / 16;
  c.row16 = kv->Hkv * (kv->D / 8);
  c.capacity = kv->capacity;
  c.table = kv->page_table;
  c.P = kv->pages_per_seq;
  c.num_pages = kv->num_pages;
  return true;
}

bool pool_ok(const dreams_page_pool_t *pool, Pool &p) {
  if (pool == nullptr || pool->page_table == nullptr || pool->refcount == nullptr || !aligned4(pool->page_table) ||
      !aligned4(pool->refcount) || pool->B < 1 || pool->B > 65535 || pool->pages_per_seq < 1 || pool->num_pages < 1 ||
      int64_t(pool->pages_per_seq) * PAGE > INT_MAX || int64_t(pool->B) * pool->pages_per_seq > INT_MAX || pool->num_pages > INT_MAX / 2)
    return false;
  p = {pool->page_table, pool->refcount, pool->B, pool->pages_per_seq, pool->num_pages};
  return true;
}

size_t fork_layout(const Pool &p, uint8_t *ws, ForkState *f) {
  size_t at = 0;
  auto take = [&](int64_t n) {
    int32_t *x = reinterpret_cast<int32_t *>(ws + at);
    at += align_up(size_t(n) * 4, 256);
    return x;
  };
  ForkState s;
  s.head = take(FORK_HEAD);
  s.first = take(p.B);
  s.len = take(p.B);
  s.src = take(p.B);
  s.dst = take(p.B);
  s.rows = take(p.B);
  s.list = take(int64_t(FORK_CTAS) * p.B);
  s.table = take(int64_t(p.B) * p.P);
  if (f != nullptr) *f = s;
  return at;
}

}  // namespace
}  // namespace dreams

using namespace dreams;

extern "C" size_t dreams_kv_reserve_workspace_size(const dreams_page_pool_t *pool) {
  Pool p;
  if (!pool_ok(pool, p)) return 0;
  return align_up(size_t(p.B) * 4, 256) + align_up(size_t(p.num_pages) * 4, 256);
}

extern "C" dreams_status_t dreams_kv_reserve(const dreams_page_pool_t *pool, const int32_t *kv_len,
                                             const int32_t *n_new, void *workspace, size_t workspace_bytes,
                                             int32_t *status_word, dreams_stream_t stream) {
  Pool p;
  if (!pool_ok(pool, p) || kv_len == nullptr || n_new == nullptr || !aligned4(kv_len) || !aligned4(n_new))
    return DREAMS_ERR_INVALID_ARG;
  if (workspace == nullptr || !aligned16(workspace) || workspace_bytes < dreams_kv_reserve_workspace_size(pool))
    return DREAMS_ERR_WORKSPACE;
  int32_t *start = static_cast<int32_t *>(workspace);
  int32_t *list = start + align_up(size_t(p.B) * 4, 256) / 4;
  kv_reserve_kernel<<<1, BOOK_THREADS, 0, reinterpret_cast<cudaStream_t>(stream)>>>(p, kv_len, n_new, start, list,
                                                                                   status_word);
  return check_launch();
}

extern "C" dreams_status_t dreams_kv_release(const dreams_page_pool_t *pool, const int32_t *begin, const int32_t *end,
                                             int32_t *status_word, dreams_stream_t stream) {
  Pool p;
  if (!pool_ok(pool, p) || begin == nullptr || end == nullptr || !aligned4(begin) || !aligned4(end))
    return DREAMS_ERR_INVALID_ARG;
  kv_release_kernel<<<dim3(unsigned((p.P + 255) / 256), unsigned(p.B)), 256, 0,
                      reinterpret_cast<cudaStream_t>(stream)>>>(p, begin, end, status_word);
  return check_launch();
}

extern "C" size_t dreams_kv_fork_workspace_size(const dreams_page_pool_t *pool) {
  Pool p;
  if (!pool_ok(pool, p)) return 0;
  return fork_layout(p, nullptr, nullptr);
}

extern "C" dreams_status_t dreams_kv_fork(const dreams_kv_cache_t *kv, const dreams_page_pool_t *pool,
                                          const int32_t *parent, const int32_t *kv_len, int32_t *new_kv_len,
                                          void *workspace, size_t workspace_bytes, int32_t *status_word,
                                          dreams_stream_t stream) {
  Pool p;
  Cache c;
  if (!pool_ok(pool, p) || !cache_ok(kv, c) || parent == nullptr || kv_len == nullptr || new_kv_len == nullptr ||
      !aligned4(parent) || !aligned4(kv_len) || !aligned4(new_kv_len))
    return DREAMS_ERR_INVALID_ARG;
  if (c.table != p.table || c.P != p.P || c.num_pages != p.num_pages) return DREAMS_ERR_INVALID_ARG;
  if (workspace == nullptr || !aligned16(workspace) || workspace_bytes < dreams_kv_fork_workspace_size(pool))
    return DREAMS_ERR_WORKSPACE;
  ForkState f;
  fork_layout(p, static_cast<uint8_t *>(workspace), &f);
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  kv_fork_table_kernel<<<FORK_CTAS, BOOK_THREADS, 0, s>>>(p, parent, kv_len, new_kv_len, f, status_word);
  const dreams_status_t st = check_launch();
  if (st != DREAMS_OK) return st;
  const int pieces = (PAGE * c.row16 + COPY_PIECE - 1) / COPY_PIECE;
  const int64_t most = int64_t(p.B) * c.n_layers * 2 * pieces;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(std::min<int64_t>(most, int64_t(num_sms()) * 8)));
  cfg.blockDim = dim3(256);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kv_fork_copy_kernel, c, f, pieces);
  if (e != cudaSuccess) {
    set_last_cuda_error(e);
    return DREAMS_ERR_CUDA;
  }
  return check_launch();
}

extern "C" dreams_status_t dreams_kv_append(const dreams_kv_cache_t *kv, int32_t layer, const void *k_new,
                                            const void *v_new, int64_t stride_b, int64_t stride_t,
                                            const int32_t *kv_len, const int32_t *n_new, int32_t B, int32_t T_max,
                                            int32_t *status_word, dreams_stream_t stream) {
  Cache c;
  if (!cache_ok(kv, c) || layer < 0 || layer >= kv->n_layers || k_new == nullptr || v_new == nullptr ||
      kv_len == nullptr || n_new == nullptr || B < 1 || B > 65535 || T_max < 1 || T_max > (1 << 20) ||
      !aligned16(k_new) || !aligned16(v_new) || !aligned4(kv_len) || !aligned4(n_new))
    return DREAMS_ERR_INVALID_ARG;
  if (B == 1) stride_b = stride_t;  // not used
  const int64_t row = int64_t(kv->Hkv) * kv->D;
  if (stride_t < row || stride_b < row || stride_t % 8 != 0 || stride_b % 8 != 0 || stride_t >= (int64_t(1) << 38) ||
      stride_b >= (int64_t(1) << 38))
    return DREAMS_ERR_INVALID_ARG;
  const int64_t blocks = (int64_t(T_max) * c.row16 + 256 * APPEND_UNROLL - 1) / (256 * APPEND_UNROLL);
  if (blocks > INT_MAX) return DREAMS_ERR_UNSUPPORTED;
  c.k += layer * c.layer16;
  c.v += layer * c.layer16;
  kv_append_kernel<<<dim3(unsigned(blocks), unsigned(B)), 256, 0, reinterpret_cast<cudaStream_t>(stream)>>>(
      c, static_cast<const uint4 *>(k_new), static_cast<const uint4 *>(v_new), stride_b / 8, stride_t / 8, kv_len, n_new,
      T_max, status_word);
  return check_launch();
}

extern "C" dreams_status_t dreams_kv_prune(const dreams_kv_cache_t *kv, int32_t B, const int32_t *keep, int32_t v0,
                                           int32_t n_vis, int32_t r, const int32_t *kv_len, const int32_t *refcount,
                                           int32_t *new_kv_len, int32_t *status_word, dreams_stream_t stream) {
  Cache c;
  if (!cache_ok(kv, c) || B < 1 || B > 65535 || kv_len == nullptr || new_kv_len == nullptr || new_kv_len == kv_len ||
      v0 < 0 || n_vis < 0 || r < 0 || r > n_vis || (keep == nullptr && r > 0) || !aligned4(keep) || !aligned4(kv_len) ||
      !aligned4(new_kv_len) || !aligned4(refcount))
    return DREAMS_ERR_INVALID_ARG;
  if (int64_t(c.n_layers) * 2 * c.row16 > INT_MAX) return DREAMS_ERR_UNSUPPORTED;
  // The widest column block that still gives every SM two CTAs: wide blocks
  // read whole lines of a slot, narrow ones put more of a small cache in flight.
  const int64_t lanes = int64_t(c.n_layers) * 2 * B, want = 2 * int64_t(num_sms());
  int cw = 32;
  while (cw > 4 && lanes * ((c.row16 + cw - 1) / cw) < want) cw /= 2;
  const dim3 grid(unsigned(int64_t(c.n_layers) * 2 * ((c.row16 + cw - 1) / cw)), unsigned(B));
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  auto *kernel = cw == 32 ? kv_prune_kernel<32> : cw == 16 ? kv_prune_kernel<16> : cw == 8 ? kv_prune_kernel<8> : kv_prune_kernel<4>;
  kernel<<<grid, PRUNE_THREADS, 0, s>>>(c, keep, v0, n_vis, r, kv_len, refcount, new_kv_len, status_word);
  return check_launch();
}
