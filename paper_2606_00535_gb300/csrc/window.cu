// window.cu -- attention with a sliding window and sinks.
//
// Query t of a sequence with L committed slots is at position p = L + t (causal)
// or L + depth(t) (draft tree) and sees slot s when p - s < window or s < sinks,
// new slots only up to its own (causal) or along its ancestors (tree). The keys a
// block of query rows can see are two runs of slots, the sinks and the window of
// its first query up to its last one; the kernel numbers them 0 .. n-1 as one list,
// so sinks and window share tiles and nothing between them is read.
//
// Few rows (at most 16 of a KV head: single tokens, short drafts), bound by reading K
// and V once. A CTA takes part of the key list of a sequence and KV head; its four
// warps take 16-key tiles in turn, each with its own ring of cp.async stages, so no
// barrier stands in the stream. Scores and P V run on m16n8k16 tensor instructions
// (16 rows are all there are: the fifth-generation ones would work on 128), with the
// running maximum and sum of each row in f32 registers. Where the lists are few, each
// is split over a cluster, whose CTAs push their parts into each other's shared memory
// and join them there, in list order. More rows go to window_tc.cu. Head dim 128: 64
// sequences of 8 KV heads, window 4096, 161 us, 95% of the copy rate; one of 4, window
// 1024, 6.3 us, a chain of dependent loads.
//
// P enters P V as bf16, which makes the outputs' error against 64 bits 1.2 to 1.4 times
// that of f32 probabilities. With at most 8 rows (FOLD) half of an instruction's 16 is
// free: it takes what is left of P, and the halves are added at the end, so that 16 bits
// of P count. With 9 to 16 rows that would be a second product (the batch above 171 us
// with one), so there P is one bf16, as in window_tc.cu.
#include <limits.h>
#include <math.h>

#include <algorithm>

#include "rows.cuh"

namespace dreams {
namespace {

using namespace win;

constexpr int KT = 16;    // keys of a warp's tile

template <int D>
struct RowsCfg {
  static constexpr int STAGES = D == 128 ? 3 : 6;
  static constexpr int ROW = D * 2;                // bytes of a key
  static constexpr int TILE = KT * ROW;            // K or V of a tile
  static constexpr int WARP_BYTES = STAGES * 2 * TILE;
  static constexpr int RING = WARPS * WARP_BYTES;  // afterwards the warps' outputs [WARPS][16][D] f32
  static constexpr int SMEM = RING + RB * D * 4;   // and what the CTAs of a cluster push here
  static_assert(RING >= WARPS * RB * D * 4, "partials fit");
};

// Attention of the rows over keys [i0, i1) of the list. Afterwards sh.ml holds each
// warp's (m, l) per row, and `ring` its unnormalised outputs [warp][row][D] in f32.
template <int D, bool FOLD>
__device__ __forceinline__ void stream_keys(const WinParams &p, RowsShared &sh, uint8_t *smem, const KeyList &kl, int b, int g, int L, int T,
                                            int i0, int i1) {
  using C = RowsCfg<D>;
  constexpr int CH = D / 8;         // 16-byte columns of a key
  constexpr int H = FOLD ? 1 : 2;  // rows of a thread
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int ntiles = (i1 - i0 + KT - 1) / KT;

  // this warp's tiles: warp, warp + WARPS, ...
  const uint32_t ring = smem_u32(smem) + warp * C::WARP_BYTES;
  const int my = ntiles > warp ? (ntiles - warp + WARPS - 1) / WARPS : 0;
  // lane k (mod 16) looks after key k of a tile: its slot and page entry one
  // tile ahead of the copy
  int nslot = -1, npage = 0;
  auto look = [&](int j) {
    const int i = i0 + (warp + j * WARPS) * KT + (lane & 15);
    nslot = j < my && i < i1 ? kl.slot(i) : -1;
    if (p.table != nullptr && nslot >= 0) npage = p.table[int64_t(b) * p.P + (nslot >> 6)];
  };
  // Copies of 16 bytes: lanes CH to a key, 32 / CH keys at a time. A key is known by
  // its row (slot and page, without the head): below 2^32 in any memory.
  constexpr uint32_t NO_ROW = 0xffffffffu;
  const int ch = lane % CH;
  const int64_t pitch = int64_t(p.Hkv) * D;
  const __nv_bfloat16 *kp = p.k + int64_t(g) * D + ch * 8, *vp = p.v + int64_t(g) * D + ch * 8;
  auto issue = [&](int j, uint32_t st) {
    if (j < my) {
      uint32_t at = NO_ROW;
      if (nslot >= 0) {
        if (p.table == nullptr) {
          at = uint32_t(b) * uint32_t(p.capacity) + uint32_t(nslot);
        } else if (npage >= 0 && npage < p.num_pages) {
          at = uint32_t(npage) * 64u + uint32_t(nslot & 63);
        } else if (lane < 16) {
          flag(p.status, DREAMS_DATA_BAD_PAGE);
        }
      }
      look(j + 1);
#pragma unroll
      for (int it = 0; it < KT * CH / 32; ++it) {
        const int key = it * (32 / CH) + lane / CH;
        const uint32_t row = __shfl_sync(0xffffffffu, at, key);
        const uint32_t dst = st + key * C::ROW + ((ch ^ (key & 7)) << 4);
        const int64_t e = row == NO_ROW ? 0 : row * pitch;
        const int bytes = row == NO_ROW ? 0 : 16;
        cp_async16(dst, kp + e, bytes);
        cp_async16(dst + C::TILE, vp + e, bytes);
      }
    }
    cp_commit();
  };
  look(0);

  // this thread's part of Q: rows lane / 4 and (H = 2) lane / 4 + 8
  const int r0 = lane >> 2, c0 = (lane & 3) * 2;
  uint32_t qf[D / 16][4];
  int off[H];
  unsigned long long anc[H];
#pragma unroll
  for (int h = 0; h < H; ++h) {
    const int r = r0 + 8 * h, t = r / p.G;
    off[h] = t < T ? t : -1;
    anc[h] = 0ull;
    if (p.parent != nullptr) {
      off[h] = sh.row[r].off;
      anc[h] = sh.row[r].anc;
    }
    const __nv_bfloat16 *src = p.q + b * p.sb + t * p.st + int64_t(g * p.G + r - t * p.G) * D + c0;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      qf[kk][h] = t < T ? *reinterpret_cast<const uint32_t *>(src + kk * 16) : 0u;
      qf[kk][h + 2] = t < T ? *reinterpret_cast<const uint32_t *>(src + kk * 16 + 8) : 0u;
      if (FOLD) qf[kk][1] = qf[kk][3] = 0u;
    }
  }
  float o[D / 8][4];
#pragma unroll
  for (int n = 0; n < D / 8; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;
  float m[H], l[H];
#pragma unroll
  for (int h = 0; h < H; ++h) {
    m[h] = -INFINITY;
    l[h] = 0.f;
  }

  const int off_max = T - 1;
  uint32_t st_in = ring, st = ring;  // the stages of the copy and of the tile
  // (one copy of the code for the ramp and the stream: a short call runs it cold)
#pragma unroll 1
  for (int j = 1 - C::STAGES; j < my; ++j) {
    if (j >= 0) {
      cp_wait<C::STAGES - 2>();
      __syncwarp();
    }
    issue(j + C::STAGES - 1, st_in);
    st_in = st_in + 2 * C::TILE == ring + C::WARP_BYTES ? ring : st_in + 2 * C::TILE;
    if (j < 0) continue;
    const int ib = i0 + (warp + j * WARPS) * KT;

    // scores: two 8-key column blocks
    float s[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
    {
      const int key = ((lane >> 4) << 3) + (lane & 7), half = (lane >> 3) & 1;
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk) {
        uint32_t kb[4];
        ldsm4(st + key * C::ROW + (((2 * kk + half) ^ (key & 7)) << 4), kb);
        mma16816(s[0], qf[kk], kb[0], kb[1]);
        mma16816(s[1], qf[kk], kb[2], kb[3]);
      }
    }
    // does every row see every key of the tile?
    const int sl = kl.slot(ib + KT - 1);
    const bool all = ib + KT <= i1 &&
                     (ib + KT <= kl.S1 ||
                      (ib >= kl.S1 && int64_t(L) + off_max - kl.slot(ib) < p.window &&
                       (p.parent != nullptr ? sl < L : sl <= L)));
    if (!all) {
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < 2 * H; ++e) {
          const int i = ib + n * 8 + c0 + (e & 1);
          if (i >= i1 || off[e >> 1] < 0 || !sees(p, L, off[e >> 1], anc[e >> 1], kl.slot(i))) s[n][e] = -INFINITY;
        }
    }
    uint32_t pf[4];
    float mx[H];
#pragma unroll
    for (int h = 0; h < H; ++h) mx[h] = fmaxf(fmaxf(s[0][2 * h], s[0][2 * h + 1]), fmaxf(s[1][2 * h], s[1][2 * h + 1]));
#pragma unroll
    for (int k = 1; k < 4; k <<= 1)
#pragma unroll
      for (int h = 0; h < H; ++h) mx[h] = fmaxf(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], k));
#pragma unroll
    for (int h = 0; h < H; ++h) mx[h] = fmaxf(m[h], mx[h] * p.scale_log2);
    if (__any_sync(0xffffffffu, mx[0] > m[0] || mx[H - 1] > m[H - 1])) {
#pragma unroll
      for (int h = 0; h < H; ++h) {
        const float corr = mx[h] == m[h] ? 1.f : tc::ex2(m[h] - mx[h]);  // (also where both are -inf)
        m[h] = mx[h];
        l[h] *= corr;
#pragma unroll
        for (int n = 0; n < D / 8; ++n) {
          o[n][2 * h] *= corr;
          o[n][2 * h + 1] *= corr;
          if (FOLD) {
            o[n][2] *= corr;
            o[n][3] *= corr;
          }
        }
      }
    }
#pragma unroll
    for (int h = 0; h < H; ++h) {
      const float nm = m[h] == -INFINITY ? 0.f : -m[h];
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const float p0 = tc::ex2(fmaf(s[n][2 * h], p.scale_log2, nm));
        const float p1 = tc::ex2(fmaf(s[n][2 * h + 1], p.scale_log2, nm));
        l[h] += p0 + p1;
        if (FOLD) {
          const uint32_t hi = __byte_perm(__float_as_uint(p0), __float_as_uint(p1), 0x7632);
          pf[2 * n] = hi;
          // (what is left may be zero, and zero times an infinity in V a NaN: 2^-20 of P is below its error)
          pf[2 * n + 1] = pack_bf16x2(fmaxf(p0 - __uint_as_float(hi << 16), p0 * 0x1p-20f),
                                      fmaxf(p1 - __uint_as_float(hi & 0xffff0000u), p1 * 0x1p-20f));
        } else {
          pf[2 * n + h] = pack_bf16x2(p0, p1);
        }
      }
    }
    // O += P V
    const int vkey = (((lane >> 3) & 1) << 3) + (lane & 7), vhalf = lane >> 4;
    const uint32_t vrow = st + C::TILE + vkey * C::ROW;
    // 0 x inf and 0 x NaN are NaN: where a key that not every row sees holds one, each
    // row takes its product from its own keys alone
    bool odd = false;
    if (!all) {
      uint32_t acc = 0;  // sums of 0 x V: zero, or NaN
#pragma unroll 2
      for (int c = 0; c < C::TILE / 512; ++c) {
        uint32_t u[4];
        asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];"
                     : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3])
                     : "r"(st + C::TILE + c * 512 + lane * 16));
#pragma unroll
        for (int e = 0; e < 4; ++e) asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(acc) : "r"(u[e]), "r"(0u));
      }
      odd = __any_sync(0xffffffffu, (acc & 0x7fff7fffu) != 0u);
    }
    if (__builtin_expect(!odd, 1)) {
#pragma unroll
      for (int n = 0; n < D / 8; n += 2) {
        uint32_t vb[4];
        ldsm4t(vrow + (((n + vhalf) ^ (vkey & 7)) << 4), vb);
        mma16816(o[n], pf, vb[0], vb[1]);
        mma16816(o[n + 1], pf, vb[2], vb[3]);
      }
    } else {
#pragma unroll 1
      for (int r = 0; r < 8 * H; ++r) {
        const RowInfo ri = sh.row[r];
        uint32_t keep[2];
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
          keep[hh] = 0u;
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int i = ib + hh * 8 + c0 + e;
            if (i < i1 && ri.off >= 0 && sees(p, L, ri.off, ri.anc, kl.slot(i))) keep[hh] |= 0xffffu << (16 * e);
          }
        }
#pragma unroll
        for (int n = 0; n < D / 8; n += 2) {
          uint32_t vb[4];
          ldsm4t(vrow + (((n + vhalf) ^ (vkey & 7)) << 4), vb);
          float a0[4] = {0.f, 0.f, 0.f, 0.f}, a1[4] = {0.f, 0.f, 0.f, 0.f};
          mma16816(a0, pf, vb[0] & keep[0], vb[1] & keep[1]);
          mma16816(a1, pf, vb[2] & keep[0], vb[3] & keep[1]);
#pragma unroll
          for (int h = 0; h < 2; ++h)
            if (r0 + (FOLD ? 0 : 8 * h) == r) {
              o[n][2 * h] += a0[2 * h];
              o[n][2 * h + 1] += a0[2 * h + 1];
              o[n + 1][2 * h] += a1[2 * h];
              o[n + 1][2 * h + 1] += a1[2 * h + 1];
            }
        }
      }
    }
    st = st + 2 * C::TILE == ring + C::WARP_BYTES ? ring : st + 2 * C::TILE;
  }
  cp_wait<0>();
  __syncthreads();  // the stages are free

  float *so = reinterpret_cast<float *>(smem);
#pragma unroll
  for (int h = 0; h < H; ++h) {
    l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
    l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
    const int r = r0 + 8 * h;
    if ((lane & 3) == 0) sh.ml[warp][r] = make_float2(m[h], l[h]);
    if (off[h] >= 0) {
#pragma unroll
      for (int n = 0; n < D / 8; ++n)
        *reinterpret_cast<float2 *>(so + (warp * RB + r) * D + n * 8 + c0) =
            FOLD ? make_float2(o[n][0] + o[n][2], o[n][1] + o[n][3]) : make_float2(o[n][2 * h], o[n][2 * h + 1]);
    }
  }
  __syncthreads();
}

template <int D, bool FOLD>
__global__ void __launch_bounds__(32 * WARPS) window_rows_kernel(const WinParams p) {
  using C = RowsCfg<D>;
  extern __shared__ __align__(1024) uint8_t smem[];
  __shared__ RowsShared sh;
  const int tid = threadIdx.x;
  int x = blockIdx.x;
  const int split = x % p.nsplit;
  x /= p.nsplit;
  const int g = x % p.Hkv, b = x / p.Hkv;
  if (p.nsplit > 1) cluster_arrive();  // this CTA runs: it may be written to
  after_previous();
  const int T = p.q_len[b], L = p.kv_len[b];
  const bool report = split == 0 && g == 0;
  int bad = 0;
  if (T < 0 || T > p.T_max) bad = DREAMS_DATA_BAD_TREE_LEN;
  else if (L < 0 || int64_t(L) + T > p.capacity) bad = DREAMS_DATA_BAD_KV_LEN;
  if (bad && report && tid == 0) flag(p.status, bad);
  // (all CTAs of a cluster come to the same answer; none leaves while it may be written to)
  if (bad || T == 0 || !load_rows(p, sh, b, L, T, report)) {
    if (p.nsplit > 1) cluster_wait();
    return;
  }
  const KeyList kl = key_list(p, L, 0, T - 1);
  const int64_t per = ((int64_t(kl.n) + p.nsplit - 1) / p.nsplit + KT - 1) / KT * KT;
  const int i0 = int(::min(int64_t(kl.n), split * per)), i1 = int(::min(int64_t(kl.n), i0 + per));
  stream_keys<D, FOLD>(p, sh, smem, kl, b, g, L, T, i0, i1);
  finish_rows<D>(p, sh, smem, C::RING, b, g, T, split);
}

// ------------------------------------------------------------------ host side
// CTAs of a list: as many as still run at the same time, two to an SM. One CTA takes
// 14 us for 1024 keys whatever else runs; with all places taken the copies are bound by
// HBM, and further splits only add joins. Measured on the GPU for 8 KV heads, window
// 4096, head dim 128, in us:
//   lists        8     64    128    512
//   1 CTA     57.5   59.6   60.4  160.5
//   2         31.8   33.8   44.6  175.7
//   4         18.4   24.4   50.2  179.7
//   8         12.0   30.7   60.2  211.9
//   16         9.7   50.0   96.9  360.6
// Keys are counted by the cache's capacity, as the lengths are on the device: a short
// sequence in a large cache gets CTAs without keys. One of 50 tokens, window 4096, takes
// 3.4 us in a cache of 64 slots and 5.4 in one of 32768, one of 300 5.1 and 5.6; from
// some thousand on, and with 64 sequences, there is no difference.
constexpr int MAX_SPLIT = 16;
int split_of(int64_t lists, int64_t keys) {
  int n = 1;
  while (n < MAX_SPLIT && lists * n * 2 <= 2 * int64_t(num_sms()) && keys / n > WARPS * KT) n *= 2;
  return n;
}

template <int D, bool FOLD>
dreams_status_t launch_rows(WinParams p, cudaStream_t stream) {
  p.nsplit = split_of(int64_t(p.B) * p.Hkv, std::min<int64_t>(p.capacity, int64_t(p.window) - 1 + p.T_max + p.sinks));
  return launch_lists<window_rows_kernel<D, FOLD>>(early_launch(), RowsCfg<D>::SMEM, int64_t(p.B) * p.Hkv, p.nsplit, stream, p);
}

}  // namespace
}  // namespace dreams

namespace dreams {
namespace win {

static bool shapes_ok(const dreams_kv_cache_t *kv, int32_t B, int32_t T_max, int32_t Hq, int32_t window, int32_t sinks,
               bool tree) {
  return kv != nullptr && B >= 1 && B <= 65535 && T_max >= 1 && T_max <= (tree ? 64 : 1 << 20) && kv->Hkv >= 1 &&
         kv->Hkv <= 65535 && Hq >= kv->Hkv && Hq % kv->Hkv == 0 && Hq / kv->Hkv <= 128 && kv->capacity >= 1 &&
         kv->n_layers >= 1 && window >= 1 && sinks >= 0;
}

dreams_status_t window_args(const void *q, int64_t q_stride_b, int64_t q_stride_t, const dreams_kv_cache_t *kv, int32_t layer, const int32_t *parent,
                            const int32_t *q_len, const int32_t *kv_len, int32_t B, int32_t T_max, int32_t Hq, float scale, int32_t window,
                            int32_t sinks, void *out, float *lse, int32_t *status_word, WinParams &p) {
  if (q == nullptr || out == nullptr || kv == nullptr || q_len == nullptr || kv_len == nullptr || kv->k == nullptr ||
      kv->v == nullptr || !shapes_ok(kv, B, T_max, Hq, window, sinks, parent != nullptr))
    return DREAMS_ERR_INVALID_ARG;
  if (kv->D != 64 && kv->D != 128) return DREAMS_ERR_UNSUPPORTED;
  if (kv->capacity > (1 << 30)) return DREAMS_ERR_UNSUPPORTED;
  if (layer < 0 || layer >= kv->n_layers || kv->layer_stride < 0) return DREAMS_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(out) || !aligned16(kv->k) || !aligned16(kv->v) || (kv->layer_stride * 2) % 16 != 0 ||
      (reinterpret_cast<uintptr_t>(lse) & 3))
    return DREAMS_ERR_INVALID_ARG;
  if (!isfinite(scale) || !(scale > 0.f)) return DREAMS_ERR_INVALID_ARG;
  if (T_max == 1) q_stride_t = int64_t(Hq) * kv->D;  // not used
  if (B == 1) q_stride_b = q_stride_t;
  if (q_stride_t < int64_t(Hq) * kv->D || q_stride_b < int64_t(Hq) * kv->D || q_stride_t % 8 != 0 ||
      q_stride_b % 8 != 0 || q_stride_t >= (int64_t(1) << 38) || q_stride_b >= (int64_t(1) << 38))
    return DREAMS_ERR_INVALID_ARG;
  if (kv->page_table != nullptr) {
    if (kv->page_size != 64) return DREAMS_ERR_UNSUPPORTED;
    if (kv->pages_per_seq < 1 || kv->num_pages < 1 || int64_t(kv->pages_per_seq) * 64 != kv->capacity)
      return DREAMS_ERR_INVALID_ARG;
  }
  p = WinParams{};
  p.q = static_cast<const __nv_bfloat16 *>(q);
  p.sb = q_stride_b;
  p.st = q_stride_t;
  p.k = static_cast<const __nv_bfloat16 *>(kv->k) + int64_t(layer) * kv->layer_stride;
  p.v = static_cast<const __nv_bfloat16 *>(kv->v) + int64_t(layer) * kv->layer_stride;
  p.out = static_cast<__nv_bfloat16 *>(out);
  p.lse = lse;
  p.table = kv->page_table;
  p.P = kv->pages_per_seq;
  p.num_pages = kv->num_pages;
  p.capacity = kv->capacity;
  p.parent = parent;
  p.q_len = q_len;
  p.kv_len = kv_len;
  p.B = B;
  p.T_max = T_max;
  p.Hq = Hq;
  p.Hkv = kv->Hkv;
  p.G = Hq / kv->Hkv;
  p.window = window;
  p.sinks = sinks;
  p.scale_log2 = scale * LOG2E;
  p.status = status_word;
  return DREAMS_OK;
}

}  // namespace win
}  // namespace dreams

using namespace dreams;

extern "C" dreams_status_t dreams_window_attention(const void *q, int64_t q_stride_b, int64_t q_stride_t,
                                                   const dreams_kv_cache_t *kv, int32_t layer, const int32_t *parent,
                                                   const int32_t *q_len, const int32_t *kv_len, int32_t B,
                                                   int32_t T_max, int32_t Hq, float scale, int32_t window,
                                                   int32_t sinks, void *out, float *lse, int32_t *status_word,
                                                   dreams_stream_t stream) {
  WinParams p;
  const dreams_status_t st =
      win::window_args(q, q_stride_b, q_stride_t, kv, layer, parent, q_len, kv_len, B, T_max, Hq, scale, window, sinks, out, lse, status_word, p);
  if (st != DREAMS_OK) return st;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (int64_t(T_max) * p.G > RB) return launch_tc(p, kv, s);
  if (int64_t(T_max) * p.G <= 8) return kv->D == 128 ? launch_rows<128, true>(p, s) : launch_rows<64, true>(p, s);
  return kv->D == 128 ? launch_rows<128, false>(p, s) : launch_rows<64, false>(p, s);
}
