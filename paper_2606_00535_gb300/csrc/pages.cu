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

#include "cache.cuh"

namespace dreams {
namespace {

constexpr int BOOK_THREADS = 1024;
constexpr int FORK_CTAS = 8;  // one portable cluster

struct Pool {
  int32_t *table;
  int32_t *ref;
  int32_t B, P, num_pages;
};

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
// One block. `g` lanes of a warp share a row and walk its entries side by side
// (32 of them while rows are few, so that a chunk of 2048 tokens is two turns
// and not 33), counting what the row lacks; a prefix sum gives every row its
// place in the list of free pages, and a second walk fills the entries in. The
// call is a chain of about six dependent loads, whatever the pool's size up to
// some 10^4 pages: 2.4 us for one row of one entry, 2.9 us for 16 rows of up to
// 33 (12.9 with a thread per row).
struct RowSpan {
  int e0, e1, bad;  // the entries that the new tokens touch
};
__device__ __forceinline__ RowSpan row_span(const Pool &p, const int32_t *kv_len, const int32_t *n_new, int b) {
  const int64_t L = kv_len[b], n = n_new[b];
  if (L < 0 || n < 0 || L + n > int64_t(p.P) * PAGE) return {0, 0, DREAMS_DATA_BAD_KV_LEN};
  return {int(L / PAGE), n > 0 ? int((L + n + PAGE - 1) / PAGE) : int(L / PAGE), 0};
}

constexpr int LIST_SHARED = 4096;
__global__ void __launch_bounds__(BOOK_THREADS) kv_reserve_kernel(const Pool p, const int32_t *kv_len,
                                                                  const int32_t *n_new, int32_t *start,
                                                                  int32_t *list_ws, int32_t *status, int g) {
  __shared__ int s_warp[32], s_list[LIST_SHARED];
  after_previous();
  const int lane = threadIdx.x & (g - 1);
  const int row0 = int(threadIdx.x) / g, rows = BOOK_THREADS / g;
  const unsigned shift = (threadIdx.x & 31) & ~(g - 1);  // the row's lanes within the warp
  const unsigned mask = g == 32 ? 0xffffffffu : (1u << g) - 1;
  int base = 0;
  for (int b0 = 0; b0 < p.B; b0 += rows) {
    const int b = b0 + row0;
    int need = 0, bad = 0;
    if (b < p.B) {
      const RowSpan s = row_span(p, kv_len, n_new, b);
      bad = s.bad;
      for (int e = s.e0 + lane; e < s.e1; e += g) {
        const int pg = p.table[int64_t(b) * p.P + e];
        if (pg == -1) ++need;
        else if (pg < 0 || pg >= p.num_pages) bad |= DREAMS_DATA_BAD_PAGE;
        else if (__ldcg(p.ref + pg) != 1) bad |= DREAMS_DATA_SHARED_PAGE;
      }
    }
    __syncwarp();
    for (int o = 1; o < g; o <<= 1) {
      need += __shfl_xor_sync(0xffffffffu, need, o);
      bad |= __shfl_xor_sync(0xffffffffu, bad, o);
    }
    if (bad) {
      if (lane == 0) flag(status, bad);
      need = 0;
    }
    int total;
    const int r = base + block_scan(lane == 0 ? need : 0, s_warp, total);
    if (b < p.B && lane == 0) start[b] = need > 0 ? r : -1;
    base += total;
  }
  if (base == 0) return;
  const int want = ::min(base, p.num_pages);
  int32_t *list = want <= LIST_SHARED ? s_list : list_ws;
  const int have = list_free(p.ref, 0, p.num_pages, want, list, s_warp);
  __syncthreads();  // start[] and list[] are written
  for (int b0 = 0; b0 < p.B; b0 += rows) {
    const int b = b0 + row0;
    const int r = b < p.B ? start[b] : -1;
    int e0 = 0, e1 = 0;
    if (r >= 0) {
      const RowSpan s = row_span(p, kv_len, n_new, b);
      e0 = s.e0;
      e1 = s.e1;
    }
    int32_t *row = p.table + int64_t(b) * p.P;
    // a row gets all that it lacks or nothing
    int need = 0;
    for (int e = e0 + lane; e < e1; e += g) need += row[e] == -1;
    __syncwarp();
    for (int o = 1; o < g; o <<= 1) need += __shfl_xor_sync(0xffffffffu, need, o);
    if (r >= 0 && r + need > have) {
      if (lane == 0) flag(status, DREAMS_DATA_NO_PAGES);
      e1 = e0;
    }
    int at = r;
    for (int e = e0; __any_sync(0xffffffffu, e < e1); e += g) {
      const bool lacks = e + lane < e1 && row[e + lane] == -1;
      const unsigned who = (__ballot_sync(0xffffffffu, lacks) >> shift) & mask;
      if (lacks) {
        const int pg = list[at + __popc(who & ((1u << lane) - 1))];
        row[e + lane] = pg;
        p.ref[pg] = 1;
      }
      at += __popc(who);
    }
  }
}

// ------------------------------------------------------------------ release
// One thread per table entry: two dependent accesses, 1.3 us.
__global__ void __launch_bounds__(256) kv_release_kernel(const Pool p, const int32_t *begin, const int32_t *end,
                                                         int32_t *status) {
  after_previous();
  const int b = blockIdx.y;
  const int e = blockIdx.x * 256 + threadIdx.x;
  const int64_t lo = begin[b], hi = end[b];
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
  *at = -1;
  if (atomicSub(p.ref + pg, 1) <= 0) {  // a page that by its count nobody holds: the count stays
    atomicAdd(p.ref + pg, 1);
    flag(status, DREAMS_DATA_BAD_PAGE);
  }
}

// ------------------------------------------------------------------ fork
// The workspace.
struct ForkState {
  int32_t *head;   // [0] copies, then a word per CTA with its data flags, then one with the free pages it found
  int32_t *src, *dst, *rows;  // [B] copies: page, new page, rows of it
  int32_t *list;   // [FORK_CTAS][B] free pages by CTA
  int32_t *by_row;  // [FORK_CTAS][4][B] where the rows do not fit into shared memory
  int32_t *table;  // [B, P] the new table
};
constexpr int HEAD_FLAGS = 1, HEAD_FOUND = HEAD_FLAGS + FORK_CTAS, FORK_HEAD = HEAD_FOUND + FORK_CTAS;
constexpr int FORK_SHARED_ROWS = 2048, FORK_UNROLL = 4;
// One CTA for tables of up to so many entries: its barriers are cheaper; eight
// keep more loads in flight. Whole call with copies of one row each, us on the GPU:
//   entries    448   1024   2048   3072   4096   6144   8192  12288
//   one CTA    4.4    5.0    5.5    6.2    6.7    8.4    9.4   12.1
//   eight      5.6    6.2    6.2    6.2    6.5    6.6    6.7    7.1
constexpr int FORK_ONE_CELLS = 4096;

// (Not the .aligned forms: warps come here from loops that their lanes left at
// different turns.)
__device__ __forceinline__ void cluster_sync() {
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release;\n barrier.cluster.wait.acquire;" ::: "memory");
}

// The new table, counts and lengths, and the list of pages to copy. A chain of
// dependent loads and barriers: what concerns rows is worked out by every CTA
// for itself, so that the CTAs meet only twice, after the counts have changed
// and after the free pages have been listed. An error found there puts the
// counts back.
template <int CTAS>
__global__ void __launch_bounds__(BOOK_THREADS)
    kv_fork_table_kernel(const Pool p, const int32_t *parent, const int32_t *kv_len, int32_t *new_kv_len,
                         const ForkState f, bool full_pages, int32_t *status) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  after_previous();
  __shared__ int s_warp[32], s_bad;
  __shared__ int32_t s_rows[4 * FORK_SHARED_ROWS], s_list[CTAS == 1 ? FORK_SHARED_ROWS : 1];
  const int rank = CTAS == 1 ? 0 : int(blockIdx.x);
  const int t0 = rank * BOOK_THREADS + int(threadIdx.x);
  constexpr int nt = CTAS * BOOK_THREADS;
  const unsigned cells = unsigned(p.B) * unsigned(p.P);
  const bool near = p.B <= FORK_SHARED_ROWS;
  const int pitch = near ? FORK_SHARED_ROWS : p.B;
  int32_t *first = near ? s_rows : f.by_row + int64_t(rank) * 4 * p.B;  // the lowest row of each parent (B: none)
  int32_t *len = first + pitch, *par = len + pitch;                     // new length, parent
  int32_t *page = par + pitch;  // -1, or the row's place among the copies, then its new page

  if (threadIdx.x == 0) s_bad = 0;
  for (int b = threadIdx.x; b < p.B; b += BOOK_THREADS) first[b] = p.B;
  __syncthreads();
  {
    int bad = 0;
    for (int i = threadIdx.x; i < p.B; i += BOOK_THREADS) {
      int q = parent[i];
      if (q < -1 || q >= p.B) {
        bad |= DREAMS_DATA_BAD_INDEX;
        q = -1;
      }
      const int L = q < 0 ? 0 : __ldcg(kv_len + q);
      if (L < 0 || L > int64_t(p.P) * PAGE || (full_pages && L % PAGE != 0)) bad |= DREAMS_DATA_BAD_KV_LEN;
      if (q >= 0) atomicMin(first + q, i);
      len[i] = L;
      par[i] = q;
    }
    if (bad) atomicOr(&s_bad, bad);
  }
  __syncthreads();
  int bad = s_bad;

  // Adds `sign` for every entry that a cell gains, takes it for one that it loses.
  auto count = [&](int old, int now, int sign) {
    if (old == now) return;
    if (old >= 0 && old < p.num_pages) atomicSub(p.ref + old, sign);
    if (now >= 0 && now < p.num_pages) atomicAdd(p.ref + now, sign);
  };
  int want = 0;
  if (!bad) {
    // rows that get a copy of their parent's last page, in order
    for (int i0 = 0; i0 < p.B; i0 += BOOK_THREADS) {
      const int i = i0 + int(threadIdx.x);
      int need = 0;
      if (i < p.B) need = par[i] >= 0 && first[par[i]] != i && len[i] % PAGE != 0;
      int total;
      const int r = want + block_scan(need, s_warp, total);
      if (i < p.B) page[i] = need ? r : -1;
      want += total;
    }
    // new entries from the old table, and the counts
    int i = t0 / p.P, e = t0 - i * p.P, bad_cell = 0;
    const int di = nt / p.P, de = nt - di * p.P;
    for (unsigned x0 = t0; x0 < cells; x0 += FORK_UNROLL * nt) {
      int old[FORK_UNROLL], now[FORK_UNROLL];
      bool last[FORK_UNROLL], keep[FORK_UNROLL];  // the parent's last, partly filled entry; an entry of the new row
#pragma unroll
      for (int k = 0; k < FORK_UNROLL; ++k) {
        old[k] = now[k] = -1;
        last[k] = keep[k] = false;
        if (x0 + k * nt < cells) {
          const int q = par[i], L = len[i];
          old[k] = __ldcg(p.table + x0 + k * nt);
          if (q >= 0) {
            now[k] = __ldcg(p.table + int64_t(q) * p.P + e);
            last[k] = e == L / PAGE && L % PAGE != 0;
            keep[k] = e < L / PAGE || first[q] == i;
          }
        }
        i += di;
        e += de;
        if (e >= p.P) {
          e -= p.P;
          ++i;
        }
      }
#pragma unroll
      for (int k = 0; k < FORK_UNROLL; ++k)
        if (x0 + k * nt < cells) {
          if (old[k] < -1 || old[k] >= p.num_pages || (last[k] && now[k] < 0)) bad_cell = DREAMS_DATA_BAD_PAGE;
          if (!keep[k]) now[k] = -1;
          f.table[x0 + k * nt] = now[k];
          count(old[k], now[k], 1);
        }
    }
    if (bad_cell) atomicOr(&s_bad, bad_cell);
    __syncthreads();
    if (CTAS == 1) {
      bad = s_bad;
    } else {
      if (threadIdx.x == 0) f.head[HEAD_FLAGS + rank] = s_bad;
      cluster_sync();
#pragma unroll
      for (int c = 0; c < CTAS; ++c) bad |= __ldcg(f.head + HEAD_FLAGS + c);
    }
    if (!bad && want > 0) {
      // the free pages of each CTA's part of the pool, no more than there are copies
      const int part = (p.num_pages + CTAS - 1) / CTAS;
      const int lo = ::min(p.num_pages, rank * part);
      int32_t *list = CTAS == 1 && near ? s_list : f.list + int64_t(rank) * p.B;
      const int n = list_free(p.ref, lo, ::min(p.num_pages, lo + part), want, list, s_warp);
      int have[CTAS], all = 0;
      if (CTAS == 1) {
        have[0] = all = n;
        __syncthreads();
      } else {
        if (threadIdx.x == 0) f.head[HEAD_FOUND + rank] = n;
        cluster_sync();
#pragma unroll
        for (int c = 0; c < CTAS; ++c) {
          have[c] = __ldcg(f.head + HEAD_FOUND + c);
          all += have[c];
        }
      }
      if (want > all) {
        bad = DREAMS_DATA_NO_PAGES;
      } else {
        for (int i = threadIdx.x; i < p.B; i += BOOK_THREADS) {
          const int r = page[i];
          if (r < 0) continue;
          int c = 0, at = r;
#pragma unroll
          for (int k = 0; k + 1 < CTAS; ++k)
            if (c == k && at >= have[k]) {
              at -= have[k];
              ++c;
            }
          const int pg = CTAS == 1 ? list[at] : __ldcg(f.list + int64_t(c) * p.B + at);
          page[i] = pg;
          if (rank == 0) {
            // the row that keeps the parent's pages has the one to copy
            f.src[r] = __ldcg(f.table + int64_t(first[par[i]]) * p.P + len[i] / PAGE);
            f.dst[r] = pg;
            f.rows[r] = len[i] % PAGE;
            p.ref[pg] = 1;
          }
        }
        __syncthreads();
      }
    }
    if (bad)
      for (unsigned x = t0; x < cells; x += nt) count(__ldcg(p.table + x), __ldcg(f.table + x), -1);
  }
  if (t0 == 0) f.head[0] = bad ? 0 : want;
  if (bad) {  // nothing changes
    if (t0 == 0) flag(status, bad);
    if (new_kv_len != kv_len)
      for (int i = t0; i < p.B; i += nt) new_kv_len[i] = __ldcg(kv_len + i);
    return;
  }
  int i = t0 / p.P, e = t0 - i * p.P;
  const int di = nt / p.P, de = nt - di * p.P;
#pragma unroll 4
  for (unsigned x = t0; x < cells; x += nt) {
    int now = __ldcg(f.table + x);
    if (page[i] >= 0 && e == len[i] / PAGE) now = page[i];
    p.table[x] = now;
    i += di;
    e += de;
    if (e >= p.P) {
      e -= p.P;
      ++i;
    }
  }
  for (int i = t0; i < p.B; i += nt) new_kv_len[i] = len[i];
}

// The copies, in pieces of 256 threads x 4 x 16 bytes. A page is contiguous
// within a layer, so its first `rows` rows are one run of 16-byte columns.
// Pieces are counted with the place in the page outermost: those that a
// partly filled page has not are the last ones, and the copies of one page come
// close together, so that their source is read from L2 after the first. The
// lanes of a warp look at the CTA's next 32 pieces at once: looked up one by
// one, the chain of loads took longer than the copy (seven copies of 25 rows of
// 8 KB in 32 layers, whole call: 68 us; now 26, what reading and writing each
// copy at the copy rate takes).
constexpr int COPY_PIECE = 1024;
__global__ void __launch_bounds__(256) kv_fork_copy_kernel(const Cache c, const ForkState f, int pieces) {
  after_previous();
  const int lane = threadIdx.x & 31;
  const int64_t runs = int64_t(c.n_layers) * 2, segs = __ldcg(f.head) * runs, items = segs * pieces;
  for (int64_t x0 = blockIdx.x; x0 < items; x0 += int64_t(gridDim.x) * 32) {
    const int64_t x = x0 + int64_t(lane) * gridDim.x;
    int len = 0;
    const uint4 *src = nullptr;
    uint4 *dst = nullptr;
    if (x < items) {
      const int piece = int(x / segs);
      const int64_t seg = x - piece * segs;
      const int r = int(seg / runs), run = int(seg - r * runs);
      uint4 *base = ((run & 1) ? c.v : c.k) + (run >> 1) * c.layer16 + int64_t(piece) * COPY_PIECE;
      len = ::min(__ldcg(f.rows + r) * c.row16 - piece * COPY_PIECE, COPY_PIECE);
      src = base + int64_t(__ldcg(f.src + r)) * PAGE * c.row16;
      dst = base + int64_t(__ldcg(f.dst + r)) * PAGE * c.row16;
    }
    for (unsigned todo = __ballot_sync(0xffffffffu, len > 0); todo != 0; todo &= todo - 1) {
      const int l = __ffs(int(todo)) - 1;
      const int n = __shfl_sync(0xffffffffu, len, l);
      const uint4 *from = reinterpret_cast<const uint4 *>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(src), l));
      uint4 *to = reinterpret_cast<uint4 *>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(dst), l));
      uint4 v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (int(threadIdx.x) + 256 * i < n) v[i] = ld_stream(from + threadIdx.x + 256 * i);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (int(threadIdx.x) + 256 * i < n) to[threadIdx.x + 256 * i] = v[i];
    }
  }
}

// ------------------------------------------------------------------ append
// Units are 16-byte columns of (sequence, token); each thread moves K and V of up to
// four, all eight loads ahead of the stores. Bound by HBM: 24,400 rows of 2 KB, K and V,
// 30.9 us, 94% of the copy rate; 48 rows of 1 KB 2.8 us.
constexpr int APPEND_UNROLL = 4;
__global__ void __launch_bounds__(256) kv_append_kernel(const Cache c, const uint4 *k_new, const uint4 *v_new,
                                                        int64_t sb16, int64_t st16, const int32_t *kv_len,
                                                        const int32_t *n_new, int T_max, int32_t *status) {
  after_previous();
  const int b = blockIdx.y;
  const int n = n_new[b];
  const int64_t L = kv_len[b];
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
// read. A CTA walks one block of `cw` 16-byte columns of (layer, K or V,
// sequence); column blocks are independent. A thread has the same columns of the
// same rows of every step, PRUNE_UNROLL of them, and keeps PRUNE_STAGES steps
// on their way through its own part of shared memory; the list and the page
// table are in shared memory too, since looking them up lies between two steps'
// reads (four paged sequences of 2 KB rows, 8 layers: 98 us, 130 without).
// 1952 rows of 8 KB in 32 layers: 306 us, 98% of the copy rate. More CTAs per SM
// with narrower blocks are slower (512 threads 335 us, two of 768 per SM 325;
// three stages 373): fewer, wider streams suit the memory. A small cache is a
// chain of loads: one layer of 1 KB rows 5.5 us.
constexpr int PRUNE_THREADS = 768, PRUNE_UNROLL = 4, PRUNE_STAGES = 2;
constexpr int PRUNE_LIST = 8192, PRUNE_PAGES = 2048;  // indices kept in shared memory
constexpr int PRUNE_SMEM = PRUNE_STAGES * PRUNE_UNROLL * PRUNE_THREADS * 16 + (PRUNE_LIST + PRUNE_PAGES) * 4;
__global__ void __launch_bounds__(PRUNE_THREADS, 1) kv_prune_kernel(const Cache c, const int32_t *keep, int v0, int n_vis, int r,
                                                        const int32_t *kv_len, const int32_t *ref,
                                                        int32_t *new_kv_len, int32_t *status, int cw, int nblk) {
  extern __shared__ uint4 s_ring[];  // [PRUNE_STAGES][PRUNE_UNROLL][threads]
  constexpr int threads = PRUNE_THREADS;
  after_previous();
  int *s_list = reinterpret_cast<int *>(s_ring + PRUNE_STAGES * PRUNE_UNROLL * threads), *s_page = s_list + PRUNE_LIST;
  const int b = blockIdx.y;
  const int blk = blockIdx.x % nblk, rest = blockIdx.x / nblk;
  const bool reporter = blockIdx.x == 0 && threadIdx.x == 0;
  const int L = kv_len[b];
  const int32_t *list = keep + int64_t(b) * r;
  __shared__ int s_bad;
  if (threadIdx.x == 0) s_bad = 0;
  __syncthreads();
  int bad = 0;
  if (L > c.capacity || int64_t(v0) + n_vis > L) {
    bad = DREAMS_DATA_BAD_KV_LEN;
  } else {
    for (int i = threadIdx.x; i < r; i += threads) {
      const int s = list[i], before = i ? list[i - 1] : v0 - 1;
      if (s <= before || s >= v0 + n_vis) bad |= DREAMS_DATA_BAD_INDEX;
      if (i < PRUNE_LIST) s_list[i] = s;
    }
    if (c.table != nullptr)
      for (int e = v0 / PAGE + int(threadIdx.x); int64_t(e) * PAGE < L; e += threads) {
        const int pg = c.table[int64_t(b) * c.P + e];
        if (pg < 0 || pg >= c.num_pages) bad |= DREAMS_DATA_BAD_PAGE;
        else if (ref != nullptr && ref[pg] != 1) bad |= DREAMS_DATA_SHARED_PAGE;
        if (e - v0 / PAGE < PRUNE_PAGES) s_page[e - v0 / PAGE] = pg;
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
  const int c0 = blk * cw, width = ::min(cw, c.row16 - c0);
  const int step = PRUNE_UNROLL * threads / width;  // rows
  uint4 *base = ((rest & 1) ? c.v : c.k) + int64_t(rest >> 1) * c.layer16 + c0;
  int row[PRUNE_UNROLL], col[PRUNE_UNROLL];
#pragma unroll
  for (int j = 0; j < PRUNE_UNROLL; ++j) {
    const int u = int(threadIdx.x) + j * threads;
    row[j] = u / width;
    col[j] = u - row[j] * width;
    if (row[j] >= step) col[j] = -1;  // the rest of the division: none
  }
  const int *src_list = r <= PRUNE_LIST ? s_list : list;
  const int e0 = v0 / PAGE;
  const int *pages = c.table == nullptr ? nullptr : (L + PAGE - 1) / PAGE - e0 <= PRUNE_PAGES ? s_page : c.table + int64_t(b) * c.P + e0;
  auto offset = [&](int s) {
    if (pages == nullptr) return (int64_t(b) * c.capacity + s) * c.row16;
    return (int64_t(pages[s / PAGE - e0]) * PAGE + s % PAGE) * c.row16;
  };
  // The source slot of row i (which lands in v0 + i), -1 where nothing moves.
  auto source = [&](unsigned i) {
    if (i >= unsigned(n)) return -1;
    const int to = v0 + int(i), s = int(i) < r ? src_list[i] : to + shift;
    return s != to ? s : -1;
  };
  const uint32_t ring = smem_u32(s_ring + threadIdx.x);
  auto fetch = [&](unsigned i0, int stage) {
    if (i0 < unsigned(n)) {
#pragma unroll
      for (int j = 0; j < PRUNE_UNROLL; ++j) {
        const int s = col[j] < 0 ? -1 : source(i0 + row[j]);
        if (s >= 0)
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(ring + (stage * PRUNE_UNROLL + j) * threads * 16),
                       "l"(base + offset(s) + col[j])
                       : "memory");
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int s = 0; s < PRUNE_STAGES - 1; ++s) fetch(s * step, s);
  int stage = 0;
  for (unsigned i0 = 0; i0 < unsigned(n); i0 += step) {
    fetch(i0 + (PRUNE_STAGES - 1) * step, stage == 0 ? PRUNE_STAGES - 1 : stage - 1);
    asm volatile("cp.async.wait_group %0;" ::"n"(PRUNE_STAGES - 1) : "memory");
    __syncthreads();  // the whole step has been read
#pragma unroll
    for (int j = 0; j < PRUNE_UNROLL; ++j) {
      const unsigned i = i0 + row[j];
      if (col[j] >= 0 && source(i) >= 0) base[offset(v0 + int(i)) + col[j]] = s_ring[(stage * PRUNE_UNROLL + j) * threads + threadIdx.x];
    }
    stage = stage + 1 == PRUNE_STAGES ? 0 : stage + 1;
  }
}

// ------------------------------------------------------------------ host side
inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

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
  s.src = take(p.B);
  s.dst = take(p.B);
  s.rows = take(p.B);
  s.list = take(int64_t(FORK_CTAS) * p.B);
  s.by_row = take(p.B <= FORK_SHARED_ROWS ? 0 : int64_t(FORK_CTAS) * 4 * p.B);
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
  int g = 32;
  while (g > 1 && int64_t(p.B) * g > BOOK_THREADS) g /= 2;
  return launch(early_launch(), kv_reserve_kernel, dim3(1), BOOK_THREADS, 0, 1, stream, p, kv_len, n_new, start, list, status_word, g);
}

extern "C" dreams_status_t dreams_kv_release(const dreams_page_pool_t *pool, const int32_t *begin, const int32_t *end,
                                             int32_t *status_word, dreams_stream_t stream) {
  Pool p;
  if (!pool_ok(pool, p) || begin == nullptr || end == nullptr || !aligned4(begin) || !aligned4(end))
    return DREAMS_ERR_INVALID_ARG;
  return launch(early_launch(), kv_release_kernel, dim3(unsigned((p.P + 255) / 256), unsigned(p.B)), 256, 0, 1, stream, p, begin, end, status_word);
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
  const bool full_pages = kv == nullptr;  // there is nothing to copy
  if (!pool_ok(pool, p) || (!full_pages && !cache_ok(kv, c)) || parent == nullptr || kv_len == nullptr || new_kv_len == nullptr ||
      !aligned4(parent) || !aligned4(kv_len) || !aligned4(new_kv_len))
    return DREAMS_ERR_INVALID_ARG;
  if (!full_pages && (c.table != p.table || c.P != p.P || c.num_pages != p.num_pages)) return DREAMS_ERR_INVALID_ARG;
  if (workspace == nullptr || !aligned16(workspace) || workspace_bytes < dreams_kv_fork_workspace_size(pool))
    return DREAMS_ERR_WORKSPACE;
  ForkState f;
  fork_layout(p, static_cast<uint8_t *>(workspace), &f);
  const bool one = int64_t(p.B) * p.P <= FORK_ONE_CELLS;
  const dreams_status_t st = launch(early_launch(), one ? kv_fork_table_kernel<1> : kv_fork_table_kernel<FORK_CTAS>, dim3(one ? 1 : FORK_CTAS), BOOK_THREADS, 0,
                                    one ? 1 : FORK_CTAS, stream, p, parent, kv_len, new_kv_len, f, full_pages, status_word);
  if (st != DREAMS_OK || full_pages) return st;
  const int pieces = (PAGE * c.row16 + COPY_PIECE - 1) / COPY_PIECE;
  const int64_t most = int64_t(p.B) * c.n_layers * 2 * pieces;
  return launch(early_launch(), kv_fork_copy_kernel, dim3(unsigned(std::min<int64_t>(most, int64_t(num_sms()) * 8))), 256, 0, 1, stream, c, f, pieces);
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
  const int64_t row = int64_t(kv->Hkv) * kv->D;
  if (T_max == 1) stride_t = row;  // not used
  if (B == 1) stride_b = stride_t;
  if (stride_t < row || stride_b < row || stride_t % 8 != 0 || stride_b % 8 != 0 || stride_t >= (int64_t(1) << 38) ||
      stride_b >= (int64_t(1) << 38))
    return DREAMS_ERR_INVALID_ARG;
  const int64_t blocks = (int64_t(T_max) * c.row16 + 256 * APPEND_UNROLL - 1) / (256 * APPEND_UNROLL);
  if (blocks > INT_MAX) return DREAMS_ERR_UNSUPPORTED;
  c.k += layer * c.layer16;
  c.v += layer * c.layer16;
  return launch(early_launch(), kv_append_kernel, dim3(unsigned(blocks), unsigned(B)), 256, 0, 1, stream, c, static_cast<const uint4 *>(k_new),
                static_cast<const uint4 *>(v_new), stride_b / 8, stride_t / 8, kv_len, n_new, T_max, status_word);
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
  // A CTA takes an SM. Blocks as wide as still fill the SMs once; or, where that
  // leaves over a quarter of them idle in the last round, the first narrower ones
  // that do not, down to 512 bytes (192 walks: 3 blocks 175 us, one 209).
  const int64_t walks = int64_t(c.n_layers) * 2 * B, sms = num_sms();
  int nblk = int(std::max<int64_t>(1, std::min<int64_t>((c.row16 + 1) / 2, sms / walks)));
  for (int n = nblk; n <= 8 && c.row16 / n >= 32; ++n) {
    const int64_t ctas = walks * n;
    if (ctas * 4 >= (ctas + sms - 1) / sms * sms * 3) {
      nblk = n;
      break;
    }
  }
  int cw = (c.row16 + nblk - 1) / nblk;
  const int unit = cw >= 32 ? 8 : 2;  // whole sectors, whole lines where blocks are wide
  cw = std::min((cw + unit - 1) / unit * unit, PRUNE_UNROLL * PRUNE_THREADS);
  nblk = (c.row16 + cw - 1) / cw;
  const dreams_status_t st = ensure_max_dynamic_smem(reinterpret_cast<const void *>(kv_prune_kernel), PRUNE_SMEM);
  if (st != DREAMS_OK) return st;
  const dim3 grid(unsigned(int64_t(c.n_layers) * 2 * nblk), unsigned(B));
  return launch(early_launch(), kv_prune_kernel, grid, PRUNE_THREADS, PRUNE_SMEM, 1, stream, c, keep, v0, n_vis, r, kv_len, refcount, new_kv_len, status_word, cw,
                nblk);
}
