// kv8_attn.cu -- attention over a cache whose full pages are held in 8 bits.
//
// Few rows (at most 16 of a KV head: single tokens, short drafts), bound by reading K
// and V once. As in window.cu, a CTA takes part of the keys of a sequence and KV head, its
// warps take tiles in turn, each with its own ring of cp.async stages, scores and P V run
// on m16n8k16 tensor instructions, and a cluster's CTAs join their parts in shared
// memory. What differs is the tiles. Keys come in runs, the sinks and the window, each
// of them first in 8 bits, then in bf16; a tile is 32 codes' or 16 bf16 keys, which take
// the same bytes of a stage, lies in one page, and has one power of K and one of V.
// Codes become bf16 on their way from shared memory to the tensor instructions: three
// integer instructions for two (kv8.cuh) and a product with 2^120. The power of K goes
// into the scale of the scores, that of V into P before its rounding: both exact, and
// bf16 has the range.
//   A code row's 16 bytes of ldmatrix hold dimensions 4 c .. 4 c + 3 for thread c of four,
//   where bf16 rows give 2 c, 2 c + 1 and those 8 on. Q's registers, and with them the
//   products over dimensions, follow the codes (bf16 tiles read K eight bytes at a time
//   to match). P V's columns are dimensions 16 j + 2 r and 16 j + 2 r + 1 in two
//   products for codes; before a warp's first bf16 tile, whose columns are in order,
//   its sums change places once.
// P enters P V as one bf16, or as two where half of an instruction's 16 rows is free,
// as in window.cu.
#include <limits.h>
#include <math.h>

#include <algorithm>

#include "cache.cuh"
#include "kv8.cuh"
#include "rows.cuh"

namespace dreams {
namespace {

using namespace win;

struct AttnParams {
  WinParams p;
  Kv8 c;
};

// A warp takes one query row straight from the definition, key by key.
template <int D>
__global__ void __launch_bounds__(256) kv8_plain_kernel(const AttnParams P) {
  after_previous();
  const WinParams &p = P.p;
  const int lane = threadIdx.x & 31;
  constexpr int E = D / 32;
  const int64_t r = int64_t(blockIdx.x) * 8 + (threadIdx.x >> 5);
  if (r >= int64_t(p.B) * p.T_max * p.Hq) return;
  const int h = int(r % p.Hq), t = int(r / p.Hq % p.T_max), b = int(r / p.Hq / p.T_max), g = h / p.G;
  const int T = p.q_len[b], L = p.kv_len[b], L8 = P.c.len8[b];
  const bool report = t == 0 && h == 0 && lane == 0;
  int bad = 0;
  if (T < 0 || T > p.T_max) bad = DREAMS_DATA_BAD_TREE_LEN;
  else if (L < 0 || int64_t(L) + T > p.capacity || len8_bad(P.c, L8, L)) bad = DREAMS_DATA_BAD_KV_LEN;
  int off = t;
  unsigned long long anc = 0ull;
  if (bad == 0 && p.parent != nullptr) {
    const int32_t *par = p.parent + int64_t(b) * p.T_max;
    int odd = 0;
    for (int i = lane; i < T; i += 32) odd |= i == 0 ? par[i] != -1 : (par[i] < 0 || par[i] >= i);
    if (__any_sync(0xffffffffu, odd)) bad = DREAMS_DATA_BAD_PARENT;
    else if (t < T) anc = tree_row(p, par, L, t, off);
  }
  if (bad != 0 && report) flag(p.status, bad);
  if (bad != 0 || t >= T) return;
  float q[E], o[E];
  const __nv_bfloat16 *src = p.q + b * p.sb + t * p.st + int64_t(h) * D + lane * E;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    q[i] = __bfloat162float(src[i]);
    o[i] = 0.f;
  }
  const KeyList kl = key_list(p, L, p.parent != nullptr ? 0 : t, t);
  float m = -INFINITY, l = 0.f;
  for (int i = 0; i < kl.n; ++i) {
    const int s = kl.slot(i);
    if (!sees(p, L, off, anc, s)) continue;
    float x = 0.f, v[E], fk = 1.f, fv = 1.f;
    int64_t at;
    if (s < L8) {
      const int pg = P.c.table[int64_t(b) * P.c.P + (s >> 6)];
      at = pg >= 0 && pg < P.c.num_pages ? (int64_t(pg) * 64 + (s & 63)) * p.Hkv + g : -1;
      if (at >= 0) {
        const uint32_t w = P.c.exps[int64_t(pg) * p.Hkv + g];
        fk = power(k_exp(w));
        fv = power(v_exp(w));
      }
    } else if (p.table == nullptr) {
      at = (int64_t(b) * p.capacity + s) * p.Hkv + g;
    } else {
      const int pg = p.table[int64_t(b) * p.P + (s >> 6)];
      at = pg >= 0 && pg < p.num_pages ? (int64_t(pg) * 64 + (s & 63)) * p.Hkv + g : -1;
    }
    if (at < 0 && lane == 0) flag(p.status, DREAMS_DATA_BAD_PAGE);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      float kx = 0.f;
      v[e] = 0.f;
      if (at >= 0) {
        const int64_t j = at * D + lane * E + e;
        kx = s < L8 ? code_value(P.c.k[j]) : __bfloat162float(p.k[j]);
        v[e] = (s < L8 ? code_value(P.c.v[j]) : __bfloat162float(p.v[j])) * fv;
      }
      x += q[e] * kx;
    }
#pragma unroll
    for (int k = 16; k > 0; k >>= 1) x += __shfl_xor_sync(0xffffffffu, x, k);
    x *= fk * p.scale_log2;
    if (x > m) {
      const float c = tc::ex2(m - x);
      l *= c;
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] *= c;
      m = x;
    }
    const float w = tc::ex2(x - (m == -INFINITY ? 0.f : m));
    l += w;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] += w * v[e];
  }
  const int64_t row = (int64_t(b) * p.T_max + t) * p.Hq + h;
#pragma unroll
  for (int e = 0; e < E; ++e) p.out[row * D + lane * E + e] = __float2bfloat16(o[e] / l);
  if (lane == 0 && p.lse != nullptr) p.lse[row] = (m + log2f(l)) * LN2;
}

template <int D>
struct Cfg8 {
  static constexpr int STAGES = D == 128 ? 3 : 6;
  static constexpr int ROW8 = D, ROW16 = 2 * D;  // bytes of a key
  static constexpr int TILE = 32 * ROW8;         // K or V of a tile
  static constexpr int WARP_BYTES = STAGES * 2 * TILE;
  static constexpr int RING = WARPS * WARP_BYTES;  // afterwards the warps' outputs [WARPS][16][D] f32
  static constexpr int SMEM = RING + RB * D * 4;   // and what the CTAs of a cluster push here
  static_assert(RING >= WARPS * RB * D * 4, "partials fit");
};

// The keys that a sequence's rows may see, as tiles: of 32 slots for those in 8 bits, the
// sinks' (na) and the window's, then of 16.
struct Tiles {
  int na, n8, nc, n;
  int s8, b0, c0, d0;  // end of the sinks in 8 bits; first slots of the window's and of the bf16 runs
  int lo, S1, hi, L8;
  __device__ __forceinline__ Tiles(const KeyList &kl, int L8_, int hi_) : lo(kl.lo), S1(kl.S1), hi(hi_), L8(L8_) {
    s8 = ::min(S1, L8);
    na = (s8 + 31) / 32;
    b0 = lo & ~31;
    n8 = na + (L8 > lo ? (L8 - b0 + 31) / 32 : 0);
    c0 = L8;
    nc = S1 > L8 ? (S1 - L8 + 15) / 16 : 0;
    d0 = ::max(lo, L8) & ~15;
    n = n8 + nc + (hi - d0 + 15) / 16;
  }
};
struct Tile {
  int slot, lo, hi;  // first slot; those in [lo, hi) are the tile's
  bool sink;
};
__device__ __forceinline__ Tile tile_of(const Tiles &k, int j) {
  if (j < k.na) return Tile{32 * j, 0, k.s8, true};
  if (j < k.n8) return Tile{k.b0 + 32 * (j - k.na), k.lo, k.L8, false};
  if (j < k.n8 + k.nc) return Tile{k.c0 + 16 * (j - k.n8), 0, k.S1, true};
  return Tile{k.d0 + 16 * (j - k.n8 - k.nc), k.lo, k.hi, false};
}

__device__ __forceinline__ void cp_async4(uint32_t dst, const void *src, int bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}

// The sums of a warp from the codes' columns (two products of 16 dimensions hold 16 j +
// 2 r and 16 j + 2 r + 1) to those in order (8 j' + r): thread c of four has dimensions
// 4 c .. 4 c + 3 of each 16, and gets 2 c, 2 c + 1 and those 8 on.
template <int D>
__device__ __forceinline__ void to_order(float (&o)[D / 8][4]) {
  const int lane = threadIdx.x & 31, low = (lane & ~3) | ((lane & 3) >> 1), high = low + 2;
  const bool odd = lane & 1;
#pragma unroll
  for (int j = 0; j < D / 8; j += 2)
#pragma unroll
    for (int h = 0; h < 4; h += 2) {
      const float a0 = o[j][h], b0 = o[j + 1][h], a1 = o[j][h + 1], b1 = o[j + 1][h + 1];  // dimensions 4 c, + 1, + 2, + 3
      float x0, x1;
      x0 = __shfl_sync(0xffffffffu, a0, low), x1 = __shfl_sync(0xffffffffu, a1, low);
      o[j][h] = odd ? x1 : x0;
      x0 = __shfl_sync(0xffffffffu, b0, low), x1 = __shfl_sync(0xffffffffu, b1, low);
      o[j][h + 1] = odd ? x1 : x0;
      x0 = __shfl_sync(0xffffffffu, a0, high), x1 = __shfl_sync(0xffffffffu, a1, high);
      o[j + 1][h] = odd ? x1 : x0;
      x0 = __shfl_sync(0xffffffffu, b0, high), x1 = __shfl_sync(0xffffffffu, b1, high);
      o[j + 1][h + 1] = odd ? x1 : x0;
    }
}

// New maxima of NB blocks of 8 keys' scores, P = 2^(s - m), and its sums. s is scaled
// already, -inf where a row does not see a key.
template <int D, int NB, bool FOLD>
__device__ __forceinline__ void soften(float (&s)[NB][4], float (&m)[FOLD ? 1 : 2], float (&l)[FOLD ? 1 : 2], float (&o)[D / 8][4]) {
  constexpr int H = FOLD ? 1 : 2;
  float mx[H];
#pragma unroll
  for (int h = 0; h < H; ++h) {
    mx[h] = fmaxf(s[0][2 * h], s[0][2 * h + 1]);
#pragma unroll
    for (int n = 1; n < NB; ++n) mx[h] = fmaxf(mx[h], fmaxf(s[n][2 * h], s[n][2 * h + 1]));
  }
#pragma unroll
  for (int k = 1; k < 4; k <<= 1)
#pragma unroll
    for (int h = 0; h < H; ++h) mx[h] = fmaxf(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], k));
#pragma unroll
  for (int h = 0; h < H; ++h) mx[h] = fmaxf(m[h], mx[h]);
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
    for (int n = 0; n < NB; ++n) {
      s[n][2 * h] = tc::ex2(s[n][2 * h] + nm);
      s[n][2 * h + 1] = tc::ex2(s[n][2 * h + 1] + nm);
      l[h] += s[n][2 * h] + s[n][2 * h + 1];
    }
  }
}

// P of two blocks of keys as an instruction's first operand. KEEP: what is left of P is
// never zero where P is not (zero times an infinity of V would be a NaN; 2^-20 of P is
// below its error). Codes are finite.
template <bool FOLD, bool KEEP>
__device__ __forceinline__ void operand(const float (&a)[4], const float (&b)[4], uint32_t (&pf)[4]) {
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    const float *s = n == 0 ? a : b;
    if (FOLD) {
      const uint32_t hi = __byte_perm(__float_as_uint(s[0]), __float_as_uint(s[1]), 0x7632);
      float r0 = s[0] - __uint_as_float(hi << 16), r1 = s[1] - __uint_as_float(hi & 0xffff0000u);
      if (KEEP) {
        r0 = fmaxf(r0, s[0] * 0x1p-20f);
        r1 = fmaxf(r1, s[1] * 0x1p-20f);
      }
      pf[2 * n] = hi;
      pf[2 * n + 1] = pack_bf16x2(r0, r1);
    } else {
      pf[2 * n] = pack_bf16x2(s[0], s[1]);
      pf[2 * n + 1] = pack_bf16x2(s[2], s[3]);
    }
  }
}

// Attention of the rows over tiles [j0, j1). Afterwards sh.ml holds each warp's (m, l) per
// row, and `smem` its unnormalised outputs [warp][row][D] in f32.
template <int D, bool FOLD>
__device__ __forceinline__ void stream_tiles(const AttnParams &P, RowsShared &sh, uint32_t (*s_exp)[6], uint8_t *smem, const Tiles &tl, int b, int g, int L, int T,
                                             int j0, int j1) {
  using C = Cfg8<D>;
  const WinParams &p = P.p;
  constexpr int H = FOLD ? 1 : 2;  // rows of a thread
  constexpr uint32_t UP = 0x7b807b80u;  // 2^120, twice
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t ring = smem_u32(smem) + warp * C::WARP_BYTES, exps = smem_u32(s_exp[warp]);
  const int my = j1 - j0 > warp ? (j1 - j0 - warp + WARPS - 1) / WARPS : 0;  // this warp's tiles: j0 + warp, + WARPS, ...
  // the tile that is copied next, and its page entry, one tile ahead of the copy
  Tile next{};
  bool next8 = false;
  int npage = -1;
  auto look = [&](int i) {
    const int j = j0 + warp + i * WARPS;
    if (i >= my) return;
    next = tile_of(tl, j);
    next8 = j < tl.n8;
    npage = next8 ? P.c.table[int64_t(b) * P.c.P + (next.slot >> 6)] : p.table != nullptr ? p.table[int64_t(b) * p.P + (next.slot >> 6)] : 0;
  };
  auto issue = [&](int i, uint32_t st, uint32_t ex) {
    if (i < my) {
      const int64_t pitch = int64_t(p.Hkv) * D;
      const bool has = npage >= 0 && npage < (next8 ? P.c.num_pages : p.table != nullptr ? p.num_pages : 1);
      if (!has && lane == 0) flag(p.status, DREAMS_DATA_BAD_PAGE);
      if (next8) {
        constexpr int CH = D / 16;  // 16-byte columns of a key
        const int ch = lane % CH, k0 = lane / CH;
        const int64_t row = has ? int64_t(npage) * 64 + (next.slot & 63) : 0;
        const uint8_t *kp = P.c.k + (row * p.Hkv + g) * D + ch * 16, *vp = P.c.v + (row * p.Hkv + g) * D + ch * 16;
        if (lane == 0) cp_async4(ex, P.c.exps + (has ? int64_t(npage) * p.Hkv + g : 0), has ? 4 : 0);
#pragma unroll
        for (int it = 0; it < CH; ++it) {
          const int key = it * (32 / CH) + k0;
          const int bytes = has && next.slot + key >= next.lo && next.slot + key < next.hi ? 16 : 0;
          const uint32_t dst = st + key * C::ROW8 + ((ch ^ (D == 128 ? key & 7 : (key >> 1) & 3)) << 4);
          const int64_t e = bytes != 0 ? key * pitch : 0;
          cp_async16(dst, kp + e, bytes);
          cp_async16(dst + C::TILE, vp + e, bytes);
        }
      } else {
        constexpr int CH = D / 8;
        const int ch = lane % CH, k0 = lane / CH;
        const int64_t row = p.table == nullptr ? int64_t(b) * p.capacity + next.slot : has ? int64_t(npage) * 64 + (next.slot & 63) : 0;
        const __nv_bfloat16 *kp = p.k + (row * p.Hkv + g) * D + ch * 8, *vp = p.v + (row * p.Hkv + g) * D + ch * 8;
#pragma unroll
        for (int it = 0; it < CH / 2; ++it) {
          const int key = it * (32 / CH) + k0;
          const int bytes = has && next.slot + key >= next.lo && next.slot + key < next.hi ? 16 : 0;
          const uint32_t dst = st + key * C::ROW16 + ((ch ^ (key & 7)) << 4);
          const int64_t e = bytes != 0 ? key * pitch : 0;
          cp_async16(dst, kp + e, bytes);
          cp_async16(dst + C::TILE, vp + e, bytes);
        }
      }
      look(i + 1);
    }
    cp_commit();
  };
  look(0);

  // this thread's part of Q: rows lane / 4 and (H = 2) lane / 4 + 8, dimensions 4 c .. 4 c + 3 of each 16
  const int r0 = lane >> 2, c = lane & 3;
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
    const __nv_bfloat16 *src = p.q + b * p.sb + t * p.st + int64_t(g * p.G + r - t * p.G) * D + 4 * c;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      const uint2 w = t < T ? *reinterpret_cast<const uint2 *>(src + kk * 16) : make_uint2(0u, 0u);
      qf[kk][h] = w.x;
      qf[kk][h + 2] = w.y;
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
  bool ordered = false;  // o's columns

  const int off_max = T - 1;
  int in = 0, at = 0;  // the stages of the copy and of the tile
#pragma unroll 1
  for (int i = 1 - C::STAGES; i < my; ++i) {
    if (i >= 0) {
      cp_wait<C::STAGES - 2>();
      __syncwarp();
    }
    issue(i + C::STAGES - 1, ring + in * 2 * C::TILE, exps + 4 * in);
    in = in + 1 == C::STAGES ? 0 : in + 1;
    if (i < 0) continue;
    const int j = j0 + warp + i * WARPS;
    const Tile t = tile_of(tl, j);
    const uint32_t st = ring + at * 2 * C::TILE;
    if (j < tl.n8) {
      const uint32_t w = s_exp[warp][at];
      float s[4][4] = {};
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk) {
        uint32_t kb[4];  // 8 keys each
        ldsm4(st + lane * C::ROW8 + ((kk ^ (D == 128 ? lane & 7 : (lane >> 1) & 3)) << 4), kb);
#pragma unroll
        for (int n = 0; n < 4; ++n)
          mma16816(s[n], qf[kk], mul_bf16x2(codes_x2<sel_of(0, 1)>(kb[n]), UP), mul_bf16x2(codes_x2<sel_of(2, 3)>(kb[n]), UP));
      }
      const float f = p.scale_log2 * power(k_exp(w)), fv = power(v_exp(w));
#pragma unroll
      for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int e = 0; e < 2 * H; ++e) s[n][e] *= f;
      // does every row see every key of the tile?
      if (!(t.slot >= t.lo && t.slot + 32 <= t.hi && (t.sink || int64_t(L) + off_max - t.slot < p.window))) {
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
          for (int e = 0; e < 2 * H; ++e) {
            const int slot = t.slot + n * 8 + 2 * c + (e & 1);
            if (slot < t.lo || slot >= t.hi || off[e >> 1] < 0 || !sees(p, L, off[e >> 1], anc[e >> 1], slot)) s[n][e] = -INFINITY;
          }
      }
      soften<D, 4, FOLD>(s, m, l, o);
#pragma unroll
      for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int e = 0; e < 2 * H; ++e) s[n][e] = s[n][e] == 0.f ? 0.f : s[n][e] * fv;  // (a marked page is not the rows' that do not see it)
      uint32_t p0[4], p1[4];
      operand<FOLD, false>(s[0], s[1], p0);
      operand<FOLD, false>(s[2], s[3], p1);
#pragma unroll
      for (int n = 0; n < D / 8; n += 2) {
        uint32_t vb[4];
        ldsm4t(st + C::TILE + lane * C::ROW8 + (((n >> 1) ^ (D == 128 ? lane & 7 : (lane >> 1) & 3)) << 4), vb);
        mma16816(o[n], p0, mul_bf16x2(codes_x2<sel_of(0, 2)>(vb[0]), UP), mul_bf16x2(codes_x2<sel_of(0, 2)>(vb[1]), UP));
        mma16816(o[n + 1], p0, mul_bf16x2(codes_x2<sel_of(1, 3)>(vb[0]), UP), mul_bf16x2(codes_x2<sel_of(1, 3)>(vb[1]), UP));
        mma16816(o[n], p1, mul_bf16x2(codes_x2<sel_of(0, 2)>(vb[2]), UP), mul_bf16x2(codes_x2<sel_of(0, 2)>(vb[3]), UP));
        mma16816(o[n + 1], p1, mul_bf16x2(codes_x2<sel_of(1, 3)>(vb[2]), UP), mul_bf16x2(codes_x2<sel_of(1, 3)>(vb[3]), UP));
      }
    } else {
      if (!ordered) to_order<D>(o);
      ordered = true;
      float s[2][4] = {};
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk) {
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          const int key = n * 8 + r0;
          uint32_t k0, k1;
          asm volatile("ld.shared.v2.b32 {%0,%1}, [%2];"
                       : "=r"(k0), "=r"(k1)
                       : "r"(st + key * C::ROW16 + (((2 * kk + (c >> 1)) ^ (key & 7)) << 4) + (c & 1) * 8));
          mma16816(s[n], qf[kk], k0, k1);
        }
      }
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < 2 * H; ++e) s[n][e] *= p.scale_log2;
      const bool all = t.slot >= t.lo && t.slot + 16 <= t.hi &&
                       (t.sink || (int64_t(L) + off_max - t.slot < p.window && (p.parent != nullptr ? t.slot + 15 < L : t.slot + 15 <= L)));
      if (!all) {
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int e = 0; e < 2 * H; ++e) {
            const int slot = t.slot + n * 8 + 2 * c + (e & 1);
            if (slot < t.lo || slot >= t.hi || off[e >> 1] < 0 || !sees(p, L, off[e >> 1], anc[e >> 1], slot)) s[n][e] = -INFINITY;
          }
      }
      soften<D, 2, FOLD>(s, m, l, o);
      uint32_t pf[4];
      operand<FOLD, true>(s[0], s[1], pf);
      const int vkey = lane & 15, vhalf = lane >> 4;
      const uint32_t vrow = st + C::TILE + vkey * C::ROW16;
      // 0 x inf and 0 x NaN are NaN: where a key that not every row sees holds one, each
      // row takes its product from its own keys alone
      bool odd = false;
      if (!all) {
        uint32_t acc = 0;  // sums of 0 x V: zero, or NaN
#pragma unroll 2
        for (int e = 0; e < C::TILE / 512; ++e) {
          uint32_t u[4];
          asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];"
                       : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3])
                       : "r"(st + C::TILE + e * 512 + lane * 16));
#pragma unroll
          for (int k = 0; k < 4; ++k) asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(acc) : "r"(u[k]), "r"(0u));
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
              const int slot = t.slot + hh * 8 + 2 * c + e;
              if (slot >= t.lo && slot < t.hi && ri.off >= 0 && sees(p, L, ri.off, ri.anc, slot)) keep[hh] |= 0xffffu << (16 * e);
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
    }
    at = at + 1 == C::STAGES ? 0 : at + 1;
  }
  cp_wait<0>();
  __syncthreads();  // the stages are free

  float *so = reinterpret_cast<float *>(smem);
#pragma unroll
  for (int h = 0; h < H; ++h) {
    l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
    l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
    const int r = r0 + 8 * h;
    if (c == 0) sh.ml[warp][r] = make_float2(m[h], l[h]);
    if (off[h] >= 0) {
      float *to = so + (warp * RB + r) * D;
#pragma unroll
      for (int n = 0; n < D / 8; n += 2) {
        float x[4];  // two columns of either product
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          x[e] = FOLD ? o[n][e] + o[n][2 + e] : o[n][2 * h + e];
          x[2 + e] = FOLD ? o[n + 1][e] + o[n + 1][2 + e] : o[n + 1][2 * h + e];
        }
        if (ordered) {
          *reinterpret_cast<float2 *>(to + n * 8 + 2 * c) = make_float2(x[0], x[1]);
          *reinterpret_cast<float2 *>(to + n * 8 + 8 + 2 * c) = make_float2(x[2], x[3]);
        } else {
          *reinterpret_cast<float4 *>(to + n * 8 + 4 * c) = make_float4(x[0], x[2], x[1], x[3]);
        }
      }
    }
  }
  __syncthreads();
}

template <int D, bool FOLD>
__global__ void __launch_bounds__(32 * WARPS) kv8_rows_kernel(const AttnParams P) {
  extern __shared__ __align__(1024) uint8_t smem[];
  __shared__ RowsShared sh;
  __shared__ uint32_t s_exp[WARPS][6];
  const WinParams &p = P.p;
  const int tid = threadIdx.x;
  int x = blockIdx.x;
  const int split = x % p.nsplit;
  x /= p.nsplit;
  const int g = x % p.Hkv, b = x / p.Hkv;
  if (p.nsplit > 1) cluster_arrive();  // this CTA runs: it may be written to
  after_previous();
  const int T = p.q_len[b], L = p.kv_len[b], L8 = P.c.len8[b];
  const bool report = split == 0 && g == 0;
  int bad = 0;
  if (T < 0 || T > p.T_max) bad = DREAMS_DATA_BAD_TREE_LEN;
  else if (L < 0 || int64_t(L) + T > p.capacity || len8_bad(P.c, L8, L)) bad = DREAMS_DATA_BAD_KV_LEN;
  if (bad && report && tid == 0) flag(p.status, bad);
  // (all CTAs of a cluster come to the same answer; none leaves while it may be written to)
  if (bad || T == 0 || !load_rows(p, sh, b, L, T, report)) {
    if (p.nsplit > 1) cluster_wait();
    return;
  }
  const Tiles tl(key_list(p, L, 0, T - 1), L8, L + T);
  const int per = (tl.n + p.nsplit - 1) / p.nsplit;
  const int j0 = ::min(tl.n, split * per), j1 = ::min(tl.n, j0 + per);
  stream_tiles<D, FOLD>(P, sh, s_exp, smem, tl, b, g, L, T, j0, j1);
  finish_rows<D>(p, sh, smem, Cfg8<D>::RING, b, g, T, split);
}

// ------------------------------------------------------------------ host side
constexpr int MAX_SPLIT = 16;
int split_of(int64_t lists, int64_t keys) {
  int n = 1;
  while (n < MAX_SPLIT && lists * n * 2 <= 2 * int64_t(num_sms()) && keys / n > WARPS * 32) n *= 2;
  return n;
}

template <int D, bool FOLD>
dreams_status_t launch_rows(AttnParams P, cudaStream_t stream) {
  P.p.nsplit = split_of(int64_t(P.p.B) * P.p.Hkv, std::min<int64_t>(P.p.capacity, int64_t(P.p.window) - 1 + P.p.T_max + P.p.sinks));
  return launch_lists(early_launch(), kv8_rows_kernel<D, FOLD>, Cfg8<D>::SMEM, int64_t(P.p.B) * P.p.Hkv, P.p.nsplit, stream, P);
}

}  // namespace
}  // namespace dreams

using namespace dreams;

extern "C" dreams_status_t dreams_kv8_attention(const void *q, int64_t q_stride_b, int64_t q_stride_t, const dreams_kv8_cache_t *kv8,
                                                const dreams_kv_cache_t *kv, int32_t layer, const int32_t *parent, const int32_t *q_len,
                                                const int32_t *kv_len, const int32_t *len8, int32_t B, int32_t T_max, int32_t Hq, float scale,
                                                int32_t window, int32_t sinks, void *out, float *lse, int32_t *status_word, dreams_stream_t stream) {
  AttnParams P{};
  const dreams_status_t st =
      win::window_args(q, q_stride_b, q_stride_t, kv, layer, parent, q_len, kv_len, B, T_max, Hq, scale, window, sinks, out, lse, status_word, P.p);
  if (st == DREAMS_ERR_INVALID_ARG) return st;
  if (!kv8_ok(kv8) || len8 == nullptr || !aligned4(len8) || kv8->n_layers != kv->n_layers || kv8->Hkv != kv->Hkv || kv8->D != kv->D)
    return DREAMS_ERR_INVALID_ARG;
  if (st != DREAMS_OK) return st;
  P.c.k = static_cast<const uint8_t *>(kv8->k) + layer * kv8->layer_stride;
  P.c.v = static_cast<const uint8_t *>(kv8->v) + layer * kv8->layer_stride;
  P.c.exps = reinterpret_cast<const uint32_t *>(kv8->exps) + int64_t(layer) * kv8->num_pages * kv8->Hkv;
  P.c.table = kv8->page_table;
  P.c.P = kv8->pages_per_seq;
  P.c.num_pages = kv8->num_pages;
  P.c.len8 = len8;
  const int64_t few = int64_t(T_max) * P.p.G;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (few <= 8) return kv->D == 128 ? launch_rows<128, true>(P, s) : launch_rows<64, true>(P, s);
  if (few <= RB) return kv->D == 128 ? launch_rows<128, false>(P, s) : launch_rows<64, false>(P, s);
  const int64_t rows = int64_t(B) * T_max * Hq, blocks = (rows + 7) / 8;
  if (blocks > INT_MAX) return DREAMS_ERR_UNSUPPORTED;
  return launch(early_launch(), kv->D == 128 ? kv8_plain_kernel<128> : kv8_plain_kernel<64>, dim3(unsigned(blocks)), 256, 0, 1, stream, P);
}
