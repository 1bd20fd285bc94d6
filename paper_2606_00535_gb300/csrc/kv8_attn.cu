// kv8_attn.cu -- attention over a cache whose full pages are held in 8 bits.
//
// Many rows of a KV head go to window_tc.cu: more than 32, with head dim 64 more than 64.
// Up to there they are blocks of 16 rows, each with a list of keys of its own, which the
// second block finds in L2. 8 sequences of 1000 to 8000 tokens, 8 KV heads, in us, here and
// there (in brackets: all of 4000): 20 rows 43.2 and 65.9 (42.6 and 40.9), 48 rows 55.1 and
// 67.4 (67.9 and 43.1), 64 rows 68.2 and 67.3; head dim 64, 48 rows 40.3 and 59.1 (49.2 and
// 36.6), 64 rows 50.4 and 59.1, 80 rows 70.4 and 60.2: the border lies where spread lengths gain more than
// equal ones lose. (One CTA for both blocks of 32 rows, K
// and V read once: 59.5 against 55.0, before scores were f16 products.)
//
// Few rows (single tokens, short drafts), bound by reading K and V once. As in window.cu, a
// CTA takes part of the keys of a sequence and KV head, its warps take tiles in turn, each
// with its own ring of cp.async stages, scores and P V run on m16n8k16 tensor
// instructions, and a cluster's CTAs join their parts in shared memory. What differs is
// the tiles. Keys come in runs, the sinks and the window, each of them first in 8 bits,
// then in bf16; a tile is 32 codes' or 16 bf16 keys, which take the same bytes of a stage,
// lies in one page, and has one power of K and one of V.
//   Both products are f16. One instruction makes two codes f16, exactly. Q is f16 times a
//   power of two of its row, which holds bf16's eight bits whole down to 2^-31 of the row's
//   largest value; P is f16, 11 bits of it, against the tile's own largest score and lifted by
//   2^14, so that it reaches 2^-38 of the tile's largest probability. The power of K goes into the
//   scale of the scores. That of V, and what the tile's largest probability is of the row's, which
//   f16 has no room for, scale each tile's own product as it joins the row's f32 sums: a page that
//   weighs 2^-60 counts like any other where its V is 2^80 times the others'.
//   With at most 8 rows (FOLD) the products are transposed, K Q^T and V^T P^T: keys, then
//   dimensions are the instruction's 16 rows and the rows its 8 columns, so none of it is
//   idle; P^T is turned over on the way (movmatrix). 64 sequences of 1500 to 32768 tokens 340
//   us, 362 with rows as rows; head dim 64 190, 203. (e4m3 products for the scores, Q being
//   two codes, 345 and 212; with 16 rows they take as long as two of f16 each, 34 clocks, and
//   64 sequences of four tokens 481 us, 359 now.)
//   A 16-byte piece of ldmatrix holds dimensions 4 c .. 4 c + 3 for thread c of four
//   where bf16 rows give 2 c, 2 c + 1; bf16 tiles read K eight bytes at a time to match
//   Q's loads. P V's columns are dimensions 16 j + 2 r and 16 j + 2 r + 1 in two
//   products for codes; before a warp's first bf16 tile, whose columns are in order,
//   its sums change places once.
// In bf16 tiles P is one bf16, or two with FOLD, as in window.cu.
// Bound by HBM when the GPU is full: 38 sequences of 16384 tokens, 8 KV heads of 128
// dimensions, 204 us, 94% of the copy rate (253 us with both operands made bf16 by integer
// instructions, which kept the ALU busy 47% of the time). 64 of 1500 to 32768, 340 us, 99%.
#include <limits.h>
#include <math.h>

#include <algorithm>

#include "cache.cuh"
#include "kv8.cuh"
#include "rows.cuh"

namespace dreams {
namespace {

using namespace win;

constexpr int MAX_RANKED = 128;

struct AttnParams {
  WinParams p;
  Kv8 c;
  int32_t blocks;  // of 16 rows, of a KV head
  int32_t ranked;  // sequences are taken longest first
};

template <int D, bool FOLD>
struct Cfg8 {
  // CTAs of an SM. With head dim 64 a tile is half the bytes for the same softmax, and one row
  // to a thread leaves room for four: 64 sequences of 1500 to 32768 tokens 190 us, 246 with two.
  // (With two rows: 326 and 327, and 38 equal ones 236 and 189, before scores were f16 products.)
  static constexpr int PER_SM = D == 64 && FOLD ? 4 : 2;
  static constexpr int STAGES = D == 128 || FOLD ? 3 : 6;
  static constexpr int ROW8 = D, ROW16 = 2 * D;  // bytes of a key
  static constexpr int TILE = 32 * ROW8;         // K or V of a tile
  static constexpr int WARP_BYTES = STAGES * 2 * TILE;
  static constexpr int RING = WARPS * WARP_BYTES;  // afterwards the warps' outputs [WARPS][16][D] f32
  static constexpr int SMEM = RING + RB * D * 4;  // and what the CTAs of a cluster push here
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

__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t codes_to_f16x2(uint32_t codes) {  // of the lower 16 bits
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(uint16_t(codes)));
  return r;
}
// An 8 x 8 matrix of 16-bit values, a row to four threads, transposed.
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}

// The sums of a warp from the codes' columns (two products of 16 dimensions hold 16 j +
// 2 r and 16 j + 2 r + 1) to those in order (8 j' + r): thread c of four has dimensions
// 4 c .. 4 c + 3 of each 16, and gets 2 c, 2 c + 1 and those 8 on.
template <int D, int W>
__device__ __forceinline__ void to_order(float (&o)[D / 8][W]) {
  const int lane = threadIdx.x & 31, low = (lane & ~3) | ((lane & 3) >> 1), high = low + 2;
  const bool odd = lane & 1;
#pragma unroll
  for (int j = 0; j < D / 8; j += 2)
#pragma unroll
    for (int h = 0; h < W; h += 2) {
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

// FOLD: from the transposed products' order (thread c of four has rows 2 c and 2 c + 1,
// dimensions 16 j + 2 r and 16 j + 2 r + 1) to row r, dimensions 8 j' + 2 c and + 1.
template <int D>
__device__ __forceinline__ void to_rows(float (&o)[D / 8][2], float (&m2)[2], float (&l2)[2], float &m, float &l) {
  const int lane = threadIdx.x & 31, r = lane >> 2, c = lane & 3, from = 4 * c + (r >> 1);
  const bool odd = r & 1;
#pragma unroll
  for (int j = 0; j < D / 8; j += 2) {
    float x[2][2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float a = __shfl_sync(0xffffffffu, o[j + e][0], from + 16 * h), b = __shfl_sync(0xffffffffu, o[j + e][1], from + 16 * h);
        x[h][e] = odd ? b : a;
      }
#pragma unroll
    for (int e = 0; e < 2; ++e) o[j][e] = x[0][e], o[j + 1][e] = x[1][e];
  }
  const float m0 = __shfl_sync(0xffffffffu, m2[0], r >> 1), m1 = __shfl_sync(0xffffffffu, m2[1], r >> 1);
  const float l0 = __shfl_sync(0xffffffffu, l2[0], r >> 1), l1 = __shfl_sync(0xffffffffu, l2[1], r >> 1);
  m = odd ? m1 : m0;
  l = c == 0 ? (odd ? l1 : l0) : 0.f;
}

// P = 2^(s - m) is scaled by 2^LIFT: f16 then holds it down to 2^-38 of the largest.
constexpr float LIFT = 14.f;

// What P against a tile's own maximum mt counts against the row's, m.
__device__ __forceinline__ float share(float mt, float m) { return mt == -INFINITY ? 1.f : tc::ex2(mt - m); }

// New maxima of NB blocks of 8 keys' scores, P in place of s, and its sums; mt: these keys'
// own maxima, -inf for a row that sees none of them, which P goes by with OWN. s is scaled
// already, -inf where a row does not see a key.
template <int D, int NB, int H, bool OWN>
__device__ __forceinline__ void soften(float (&s)[NB][2 * H], float (&m)[H], float (&l)[H], float (&o)[D / 8][2 * H], float (&mt)[H]) {
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
  for (int h = 0; h < H; ++h) {
    mt[h] = mx[h];
    mx[h] = fmaxf(m[h], mx[h]);
  }
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
      }
    }
  }
#pragma unroll
  for (int h = 0; h < H; ++h) {
    const float ref = OWN ? mt[h] : m[h], nm = ref == -INFINITY ? 0.f : LIFT - ref;
    float sum = OWN ? 0.f : l[h];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      s[n][2 * h] = tc::ex2(s[n][2 * h] + nm);
      s[n][2 * h + 1] = tc::ex2(s[n][2 * h + 1] + nm);
      sum += s[n][2 * h] + s[n][2 * h + 1];
    }
    l[h] = OWN ? fmaf(sum, share(mt[h], m[h]), l[h]) : sum;
  }
}

// Attention of the rows over tiles [j0, j1). Afterwards sh.ml holds each warp's (m, l) per
// row, and `smem` its unnormalised outputs [warp][row][D] in f32.
template <int D, bool FOLD>
__device__ __forceinline__ void stream_tiles(const AttnParams &P, RowsShared &sh, uint32_t (*s_exp)[6], uint8_t *smem, const Tiles &tl, int b, int g, int L, int T,
                                             int first, int j0, int j1) {
  using C = Cfg8<D, FOLD>;
  const WinParams &p = P.p;
  constexpr int H = FOLD ? 1 : 2;  // rows of a thread
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
  auto issue = [&](int i, int stage) {
    if (i < my) {
      const uint32_t st = ring + stage * 2 * C::TILE;
      const int64_t pitch = int64_t(p.Hkv) * D;
      const bool has = npage >= 0 && npage < (next8 ? P.c.num_pages : p.table != nullptr ? p.num_pages : 1);
      if (!has && lane == 0) flag(p.status, DREAMS_DATA_BAD_PAGE);
      if (next8) {
        constexpr int CH = D / 16;  // 16-byte columns of a key
        const int ch = lane % CH, k0 = lane / CH;
        const int64_t row = has ? int64_t(npage) * 64 + (next.slot & 63) : 0;
        const uint8_t *kp = P.c.k + (row * p.Hkv + g) * D + ch * 16, *vp = P.c.v + (row * p.Hkv + g) * D + ch * 16;
        if (lane == 0) cp_async4(exps + 4 * stage, P.c.exps + (has ? int64_t(npage) * p.Hkv + g : 0), has ? 4 : 0);
        // All of its keys: no looking at each (64 sequences of 1500 to 32768 tokens, one token, head
        // dim 64: 190 us for 200; four, head dim 128: 359 for 371).
        if (has && next.slot >= next.lo && next.slot + 32 <= next.hi) {
          const uint32_t dst = st + k0 * C::ROW8 + ((ch ^ (D == 128 ? k0 : k0 >> 1)) << 4);
          const int64_t rows = (32 / CH) * pitch;
          kp += k0 * pitch, vp += k0 * pitch;
#pragma unroll
          for (int it = 0; it < CH; ++it) {
            const uint32_t to = (D == 128 && (it & 1) ? dst ^ 64u : dst) + it * (32 / CH) * C::ROW8;
            cp_async16(to, kp + it * rows, 16);
            cp_async16(to + C::TILE, vp + it * rows, 16);
          }
        } else {
#pragma unroll
          for (int it = 0; it < CH; ++it) {
            const int key = it * (32 / CH) + k0;
            const int bytes = has && next.slot + key >= next.lo && next.slot + key < next.hi ? 16 : 0;
            const uint32_t dst = st + key * C::ROW8 + ((ch ^ (D == 128 ? key & 7 : (key >> 1) & 3)) << 4);
            const int64_t e = bytes != 0 ? key * pitch : 0;
            cp_async16(dst, kp + e, bytes);
            cp_async16(dst + C::TILE, vp + e, bytes);
          }
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

  const int r0 = lane >> 2, c = lane & 3;  // this thread's rows: r0 and (H = 2) r0 + 8
  auto info = [&](int h) { return sh.row[r0 + 8 * h]; };
  // its part of Q: dimensions 4 c .. 4 c + 3 of each 16
  auto src = [&](int h) -> const __nv_bfloat16 * {
    const int r = first + r0 + 8 * h, t = r / p.G;
    return t < T ? p.q + b * p.sb + t * p.st + int64_t(g * p.G + r - t * p.G) * D + 4 * c : nullptr;
  };
  float o[D / 8][2 * H];
  float m[H], l[H];
#pragma unroll
  for (int n = 0; n < D / 8; ++n)
#pragma unroll
    for (int e = 0; e < 2 * H; ++e) o[n][e] = 0.f;
#pragma unroll
  for (int h = 0; h < H; ++h) {
    m[h] = -INFINITY;
    l[h] = 0.f;
  }

  // what the rows see differs between the first token and the last
  const int off_min = first / p.G, off_max = ::min(T - 1, (first + RB - 1) / p.G);
  int in = 0, at = 0;  // the stages of the copy and of the tile
  auto step = [&](int i) {  // the tile after it is copied; this one is there
    cp_wait<C::STAGES - 2>();
    __syncwarp();
    issue(i + C::STAGES - 1, in);
    in = in + 1 == C::STAGES ? 0 : in + 1;
  };
#pragma unroll 1
  for (int i = 0; i < C::STAGES - 1; ++i) issue(i, i);
  in = C::STAGES - 1;
  // tiles in 8 bits come first
  const int my8 = ::min(my, j0 + warp < tl.n8 ? (tl.n8 - j0 - warp + WARPS - 1) / WARPS : 0);
  int i = 0;
  float m2[2] = {-INFINITY, -INFINITY}, l2[2] = {0.f, 0.f};  // FOLD: of rows 2 c and 2 c + 1
  if (my8 > 0) {
    uint32_t qf[D / 16][2 * H];  // f16
    float rq[H];                 // scale of a row's scores
#pragma unroll
    for (int h = 0; h < H; ++h) {
      const __nv_bfloat16 *from = src(h);
      uint2 w[D / 16];
      uint32_t bits = 0;
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk) {
        w[kk] = from != nullptr ? *reinterpret_cast<const uint2 *>(from + kk * 16) : make_uint2(0u, 0u);
        bits = __vmaxu2(bits, __vmaxu2(w[kk].x & 0x7fff7fffu, w[kk].y & 0x7fff7fffu));
      }
      bits = ::max(bits & 0xffffu, bits >> 16);
      bits = ::max(bits, __shfl_xor_sync(0xffffffffu, bits, 1));
      bits = ::max(bits, __shfl_xor_sync(0xffffffffu, bits, 2));
      // the largest magnitude comes to lie in [2^14, 2^15); an infinity or a NaN makes the row's scores NaN
      const int ex = ::max(int(bits >> 7), 15);
      const float up = bits >= 0x7f80u ? 0.f : __uint_as_float(uint32_t(268 - ex) << 23);
      rq[h] = bits >= 0x7f80u ? __uint_as_float(0x7fffffffu) : __uint_as_float(uint32_t(ex - 14) << 23) * p.scale_log2;
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint32_t u = e == 0 ? w[kk].x : w[kk].y;
          qf[kk][H * e + h] = pack_f16x2(__uint_as_float(u << 16) * up, __uint_as_float(u & 0xffff0000u) * up);
        }
    }
    // FOLD: the scales of rows 2 c and 2 c + 1
    const float rq2[2] = {__shfl_sync(0xffffffffu, rq[0], 8 * c), __shfl_sync(0xffffffffu, rq[0], 8 * c + 4)};
#pragma unroll 1
    for (; i < my8; ++i) {
      step(i);
      const Tile t = tile_of(tl, j0 + warp + i * WARPS);
      const uint32_t st = ring + at * 2 * C::TILE + lane * C::ROW8, swz = D == 128 ? lane & 7 : (lane >> 1) & 3;
      const uint32_t w = s_exp[warp][at];
      if constexpr (FOLD) {
        // K Q^T: e of group n is key 16 n + 8 (e >> 1) + r0 and row 2 c + (e & 1)
        float x[2][2][4] = {}, s[2][4];
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
          uint32_t k[4];
          ldsm4(st + ((kk ^ swz) << 4), k);
#pragma unroll
          for (int n = 0; n < 2; ++n) {
            const uint32_t a[4] = {codes_to_f16x2(k[2 * n]), codes_to_f16x2(k[2 * n + 1]), codes_to_f16x2(k[2 * n] >> 16), codes_to_f16x2(k[2 * n + 1] >> 16)};
            mma_f16(x[n][kk & 1], a, qf[kk][0], qf[kk][1]);
          }
        }
        const float pk = power(k_exp(w)), fv = power(v_exp(w));
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float f = rq2[h] * pk;
          if (f > 3.4e38f) f = 3.4e38f;  // (0 times infinity is a NaN)
#pragma unroll
          for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int e = h; e < 4; e += 2) s[n][e] = (x[n][0][e] + x[n][1][e]) * f;
        }
        if (!(t.slot >= t.lo && t.slot + 32 <= t.hi && (t.sink || int64_t(L) + (p.parent != nullptr ? T - 1 : off_max) - t.slot < p.window))) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const RowInfo ri = sh.row[2 * c + h];
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
              for (int e = h; e < 4; e += 2) {
                const int slot = t.slot + 16 * n + 8 * (e >> 1) + r0;
                if (slot < t.lo || slot >= t.hi || ri.off < 0 || !sees(p, L, ri.off, ri.anc, slot)) s[n][e] = -INFINITY;
              }
          }
        }
        float mt[2], mx[2];  // of the tile's keys, -inf for a row that sees none of them; with those before
#pragma unroll
        for (int h = 0; h < 2; ++h) mt[h] = fmaxf(fmaxf(s[0][h], s[0][2 + h]), fmaxf(s[1][h], s[1][2 + h]));
#pragma unroll
        for (int k = 4; k < 32; k <<= 1)
#pragma unroll
          for (int h = 0; h < 2; ++h) mt[h] = fmaxf(mt[h], __shfl_xor_sync(0xffffffffu, mt[h], k));
#pragma unroll
        for (int h = 0; h < 2; ++h) mx[h] = fmaxf(m2[h], mt[h]);
        if (__any_sync(0xffffffffu, mx[0] > m2[0] || mx[1] > m2[1])) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const float corr = mx[h] == m2[h] ? 1.f : tc::ex2(m2[h] - mx[h]);  // (also where both are -inf)
            m2[h] = mx[h];
            l2[h] *= corr;
#pragma unroll
            for (int n = 0; n < D / 8; ++n) o[n][h] *= corr;
          }
        }
        uint32_t pt[2][2];  // P, a key of the first 8 or the others to a row, transposed
        float of[2];        // what it counts, with V's power
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float nm = mt[h] == -INFINITY ? 0.f : LIFT - mt[h];
          float sum = 0.f;
#pragma unroll
          for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int e = h; e < 4; e += 2) {
              s[n][e] = tc::ex2(s[n][e] + nm);
              sum += s[n][e];
            }
          // the rows that see some of the page become NaN, however little it weighs; the others stay as they
          // are, whatever the codes
          if (__builtin_expect(v_exp(w) == DREAMS_KV8_NOT_FINITE, 0) && mt[h] != -INFINITY) sum = fv;
          const float sh = share(mt[h], m2[h]);
          of[h] = fv * sh;
          l2[h] = fmaf(sum, sh, l2[h]);
        }
        if (__builtin_expect(v_exp(w) != DREAMS_KV8_NOT_FINITE, 1)) {
#pragma unroll
          for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) pt[n][e] = transposed(pack_f16x2(s[n][2 * e], s[n][2 * e + 1]));
#pragma unroll
          for (int n = 0; n < D / 8; n += 2) {  // V^T P^T
            uint32_t vb[4], a[2][4];
            ldsm4t(st + C::TILE + (((n >> 1) ^ swz) << 4), vb);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const uint32_t y = __byte_perm(vb[k], 0u, 0x3120);  // two keys of one dimension, and of the next
              a[k >> 1][2 * (k & 1)] = codes_to_f16x2(y);
              a[k >> 1][2 * (k & 1) + 1] = codes_to_f16x2(y >> 16);
            }
            float z[4] = {};
            mma_f16(z, a[0], pt[0][0], pt[0][1]);
            mma_f16(z, a[1], pt[1][0], pt[1][1]);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[n + (e >> 1)][e & 1] = fmaf(z[e], of[e & 1], o[n + (e >> 1)][e & 1]);
          }
        }
      } else {
        float s[4][2 * H];
        {
          float x[4][4] = {};
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk) {
            uint32_t k[4];  // 8 keys each
            ldsm4(st + ((kk ^ swz) << 4), k);
#pragma unroll
            for (int n = 0; n < 4; ++n) mma_f16(x[n], qf[kk], codes_to_f16x2(k[n]), codes_to_f16x2(k[n] >> 16));
          }
          const float pk = power(k_exp(w));
#pragma unroll
          for (int h = 0; h < H; ++h) {
            float f = rq[h] * pk;
            if (f > 3.4e38f) f = 3.4e38f;  // (0 times infinity is a NaN)
#pragma unroll
            for (int n = 0; n < 4; ++n)
#pragma unroll
              for (int e = 0; e < 2; ++e) s[n][2 * h + e] = x[n][2 * h + e] * f;
          }
        }
        // does every row see every key of the tile?
        if (!(t.slot >= t.lo && t.slot + 32 <= t.hi && (t.sink || int64_t(L) + (p.parent != nullptr ? T - 1 : off_max) - t.slot < p.window))) {
#pragma unroll
          for (int h = 0; h < H; ++h) {
            const RowInfo ri = info(h);
#pragma unroll
            for (int n = 0; n < 4; ++n)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const int slot = t.slot + n * 8 + 2 * c + e;
                if (slot < t.lo || slot >= t.hi || ri.off < 0 || !sees(p, L, ri.off, ri.anc, slot)) s[n][2 * h + e] = -INFINITY;
              }
          }
        }
        float mt[H];
        soften<D, 4, H, true>(s, m, l, o, mt);
        const float fv = power(v_exp(w));
        if (__builtin_expect(v_exp(w) == DREAMS_KV8_NOT_FINITE, 0)) {
          // the rows that see some of the page become NaN, however little it weighs; the others stay as they
          // are, whatever the codes
#pragma unroll
          for (int h = 0; h < H; ++h)
            if (mt[h] != -INFINITY) l[h] = fv;
          at = at + 1 == C::STAGES ? 0 : at + 1;
          continue;
        }
        float of[H];  // what P counts, with V's power
#pragma unroll
        for (int h = 0; h < H; ++h) of[h] = fv * share(mt[h], m[h]);
        uint32_t p0[4], p1[4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          p0[h] = h < H ? pack_f16x2(s[0][2 * (h % H)], s[0][2 * (h % H) + 1]) : 0u;
          p0[h + 2] = h < H ? pack_f16x2(s[1][2 * (h % H)], s[1][2 * (h % H) + 1]) : 0u;
          p1[h] = h < H ? pack_f16x2(s[2][2 * (h % H)], s[2][2 * (h % H) + 1]) : 0u;
          p1[h + 2] = h < H ? pack_f16x2(s[3][2 * (h % H)], s[3][2 * (h % H) + 1]) : 0u;
        }
#pragma unroll
        for (int n = 0; n < D / 8; n += 2) {
          uint32_t vb[4], y[4];
          ldsm4t(st + C::TILE + (((n >> 1) ^ swz) << 4), vb);
#pragma unroll
          for (int k = 0; k < 4; ++k) y[k] = __byte_perm(vb[k], 0u, 0x3120);  // two keys of one dimension, and of the next
          float a0[4] = {}, a1[4] = {};
          mma_f16(a0, p0, codes_to_f16x2(y[0]), codes_to_f16x2(y[1]));
          mma_f16(a1, p0, codes_to_f16x2(y[0] >> 16), codes_to_f16x2(y[1] >> 16));
          mma_f16(a0, p1, codes_to_f16x2(y[2]), codes_to_f16x2(y[3]));
          mma_f16(a1, p1, codes_to_f16x2(y[2] >> 16), codes_to_f16x2(y[3] >> 16));
#pragma unroll
          for (int e = 0; e < 2 * H; ++e) {
            o[n][e] = fmaf(a0[e], of[e >> 1], o[n][e]);
            o[n + 1][e] = fmaf(a1[e], of[e >> 1], o[n + 1][e]);
          }
        }
      }
      at = at + 1 == C::STAGES ? 0 : at + 1;
    }
  }
  const bool ordered = my > my8;  // o's columns, in the end
  if constexpr (FOLD) {
#pragma unroll
    for (int k = 4; k < 32; k <<= 1)
#pragma unroll
      for (int h = 0; h < 2; ++h) l2[h] += __shfl_xor_sync(0xffffffffu, l2[h], k);
  }
  if (ordered) {
    if constexpr (FOLD) to_rows<D>(o, m2, l2, m[0], l[0]);
    else to_order<D, 2 * H>(o);
    uint32_t qf[D / 16][4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const __nv_bfloat16 *from = h < H ? src(h % H) : nullptr;
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk) {
        const uint2 w = from != nullptr ? *reinterpret_cast<const uint2 *>(from + kk * 16) : make_uint2(0u, 0u);
        qf[kk][h] = w.x;
        qf[kk][h + 2] = w.y;
      }
    }
#pragma unroll 1
    for (; i < my; ++i) {
      step(i);
      const Tile t = tile_of(tl, j0 + warp + i * WARPS);
      const uint32_t st = ring + at * 2 * C::TILE;
      const bool all = t.slot >= t.lo && t.slot + 16 <= t.hi &&
                       (t.sink || (int64_t(L) + (p.parent != nullptr ? T - 1 : off_max) - t.slot < p.window && (p.parent != nullptr ? t.slot + 15 < L : t.slot + 15 <= L + off_min)));
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
      float x[2][4] = {}, s[2][2 * H];
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk) {
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          const int key = n * 8 + r0;
          uint32_t k0, k1;
          asm volatile("ld.shared.v2.b32 {%0,%1}, [%2];"
                       : "=r"(k0), "=r"(k1)
                       : "r"(st + key * C::ROW16 + (((2 * kk + (c >> 1)) ^ (key & 7)) << 4) + (c & 1) * 8));
          mma16816(x[n], qf[kk], k0, k1);
        }
      }
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < 2 * H; ++e) s[n][e] = x[n][e] * p.scale_log2;
      if (!all) {
#pragma unroll
        for (int h = 0; h < H; ++h) {
          const RowInfo ri = info(h);
#pragma unroll
          for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int slot = t.slot + n * 8 + 2 * c + e;
              if (slot < t.lo || slot >= t.hi || ri.off < 0 || !sees(p, L, ri.off, ri.anc, slot)) s[n][2 * h + e] = -INFINITY;
            }
        }
      }
      float mt[H];
      soften<D, 2, H, false>(s, m, l, o, mt);
      uint32_t pf[4];
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        if constexpr (FOLD) {
          const uint32_t hi = __byte_perm(__float_as_uint(s[n][0]), __float_as_uint(s[n][1]), 0x7632);
          pf[2 * n] = hi;
          // (what is left may be zero, and zero times an infinity in V a NaN: 2^-20 of P is below its error)
          pf[2 * n + 1] = pack_bf16x2(fmaxf(s[n][0] - __uint_as_float(hi << 16), s[n][0] * 0x1p-20f),
                                      fmaxf(s[n][1] - __uint_as_float(hi & 0xffff0000u), s[n][1] * 0x1p-20f));
        } else {
          pf[2 * n] = pack_bf16x2(s[n][0], s[n][1]);
          pf[2 * n + 1] = pack_bf16x2(s[n][2], s[n][3]);
        }
      }
#pragma unroll 1
      for (int r = odd ? 0 : -1; r < (odd ? 8 * H : 0); ++r) {
        uint32_t keep[2] = {~0u, ~0u};
        if (r >= 0) {
          const RowInfo ri = sh.row[r];
#pragma unroll
          for (int hh = 0; hh < 2; ++hh) {
            keep[hh] = 0u;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int slot = t.slot + hh * 8 + 2 * c + e;
              if (slot >= t.lo && slot < t.hi && ri.off >= 0 && sees(p, L, ri.off, ri.anc, slot)) keep[hh] |= 0xffffu << (16 * e);
            }
          }
        }
#pragma unroll
        for (int n = 0; n < D / 8; n += 2) {
          uint32_t vb[4];
          ldsm4t(vrow + (((n + vhalf) ^ (vkey & 7)) << 4), vb);
          float a0[4] = {}, a1[4] = {};
          mma16816(a0, pf, vb[0] & keep[0], vb[1] & keep[1]);
          mma16816(a1, pf, vb[2] & keep[0], vb[3] & keep[1]);
#pragma unroll
          for (int e = 0; e < 2 * H; ++e)
            if (r < 0 || r == r0 + 8 * (e >> 1)) {
              o[n][e] += FOLD ? a0[e] + a0[2 + (e & 1)] : a0[e];
              o[n + 1][e] += FOLD ? a1[e] + a1[2 + (e & 1)] : a1[e];
            }
        }
      }
      at = at + 1 == C::STAGES ? 0 : at + 1;
    }
  }
  cp_wait<0>();
  __syncthreads();  // the stages are free

  float *so = reinterpret_cast<float *>(smem);
  if (FOLD && !ordered) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int r = 2 * c + h;
      if (r0 == 0) sh.ml[warp][r] = make_float2(m2[h] - LIFT, l2[h]);
#pragma unroll
      for (int n = 0; n < D / 8; n += 2) *reinterpret_cast<float2 *>(so + (warp * RB + r) * D + n * 8 + 2 * r0) = make_float2(o[n][h], o[n + 1][h]);
    }
    __syncthreads();
    return;
  }
#pragma unroll
  for (int h = 0; h < H; ++h) {
    l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
    l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
    const int r = r0 + 8 * h;
    if (c == 0) sh.ml[warp][r] = make_float2(m[h] - LIFT, l[h]);
    if (info(h).off >= 0) {
      float *to = so + (warp * RB + r) * D;
#pragma unroll
      for (int n = 0; n < D / 8; n += 2) {
        const float x0 = o[n][2 * h], x1 = o[n][2 * h + 1], y0 = o[n + 1][2 * h], y1 = o[n + 1][2 * h + 1];
        if (ordered) {
          *reinterpret_cast<float2 *>(to + n * 8 + 2 * c) = make_float2(x0, x1);
          *reinterpret_cast<float2 *>(to + n * 8 + 8 + 2 * c) = make_float2(y0, y1);
        } else {
          *reinterpret_cast<float4 *>(to + n * 8 + 4 * c) = make_float4(x0, y0, x1, y1);
        }
      }
    }
  }
  __syncthreads();
}

// The sequence of rank r by length, the longest first; r itself where lengths hardly
// differ. (p.B <= MAX_RANKED)
__device__ __noinline__ int by_length(const WinParams &p, int r) {
  __shared__ int4 s_len[MAX_RANKED / 4];
  __shared__ int s_at, s_low[WARPS], s_high[WARPS];
  int *len = reinterpret_cast<int *>(s_len);
  const int tid = threadIdx.x;
  int low = INT_MAX, high = INT_MIN;
  for (int i = tid; i < MAX_RANKED; i += 32 * WARPS) {
    const int x = i < p.B ? p.kv_len[i] : INT_MIN;
    len[i] = x;
    if (i < p.B) {
      low = ::min(low, x);
      high = ::max(high, x);
    }
  }
  low = __reduce_min_sync(0xffffffffu, low);
  high = __reduce_max_sync(0xffffffffu, high);
  if ((tid & 31) == 0) {
    s_low[tid >> 5] = low;
    s_high[tid >> 5] = high;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < WARPS; ++w) {
    low = ::min(low, s_low[w]);
    high = ::max(high, s_high[w]);
  }
  if (low > high - high / 8) return r;
  for (int i = tid; i < p.B; i += 32 * WARPS) {
    const int mine = len[i];
    int before = 0;
#pragma unroll 4
    for (int k = 0; 4 * k < p.B; ++k) {  // (behind the last there are only lowest values)
      const int4 x = s_len[k];
      before += int(x.x > mine || (x.x == mine && 4 * k < i)) + int(x.y > mine || (x.y == mine && 4 * k + 1 < i)) +
                int(x.z > mine || (x.z == mine && 4 * k + 2 < i)) + int(x.w > mine || (x.w == mine && 4 * k + 3 < i));
    }
    if (before == r) s_at = i;
  }
  __syncthreads();
  return s_at;
}

// (With head dim 128 the bounds ask for no CTAs beside it, which changes the code: 64
// sequences of 1500 to 32768 tokens, four new ones, 356 us for 364. Head dim 64: 270 for 261.)
template <int D, bool FOLD>
__global__ void __launch_bounds__(32 * WARPS, D == 128 ? 0 : Cfg8<D, FOLD>::PER_SM) kv8_rows_kernel(const AttnParams P) {
  extern __shared__ __align__(1024) uint8_t smem[];
  __shared__ RowsShared sh;
  __shared__ uint32_t s_exp[WARPS][6];
  const WinParams &p = P.p;
  const int tid = threadIdx.x;
  int x = blockIdx.x;
  const int split = x % p.nsplit;
  x /= p.nsplit;
  const int first = x % P.blocks * RB;  // of the KV head's rows
  x /= P.blocks;
  const int g = x % p.Hkv;
  int b = x / p.Hkv;
  if (p.nsplit > 1) cluster_arrive();  // this CTA runs: it may be written to
  after_previous();
  if (P.ranked) b = by_length(p, b);
  const int T = p.q_len[b], L = p.kv_len[b], L8 = P.c.len8[b];
  const bool report = split == 0 && g == 0 && first == 0;
  int bad = 0;
  if (T < 0 || T > p.T_max) bad = DREAMS_DATA_BAD_TREE_LEN;
  else if (L < 0 || int64_t(L) + T > p.capacity || len8_bad(P.c, L8, L)) bad = DREAMS_DATA_BAD_KV_LEN;
  if (bad && report && tid == 0) flag(p.status, bad);
  // (all CTAs of a cluster come to the same answer; none leaves while it may be written to)
  if (bad || T * p.G <= first || !load_rows(p, sh, b, L, T, report, first)) {
    if (p.nsplit > 1) cluster_wait();
    return;
  }
  const int last = ::min(T - 1, (first + RB - 1) / p.G);
  const Tiles tl(key_list(p, L, first / p.G, last), L8, L + (p.parent != nullptr ? T : last + 1));
  const int per = (tl.n + p.nsplit - 1) / p.nsplit;
  const int j0 = ::min(tl.n, split * per), j1 = ::min(tl.n, j0 + per);
  stream_tiles<D, FOLD>(P, sh, s_exp, smem, tl, b, g, L, T, first, j0, j1);
  finish_rows<D>(p, sh, smem, Cfg8<D, FOLD>::RING, b, g, T, split, first);
}

// ------------------------------------------------------------------ host side
// CTAs of a list, and the order of the lists. One CTA takes 8 us for 1000 keys whatever
// else runs, and with all places taken the copies are bound by HBM, so lists are split
// while all CTAs (`fit` places) still run at the same time, 16 to a list only while each
// has an SM of its own, and once more for several sequences of which each part keeps
// 1000 keys, as their lengths may differ.
// Where not all CTAs run at the same time, the longest sequences go first. Measured on
// the GPU for 8 KV heads, head dim 128, lengths spread from a to b, in us; (r): longest first
//   lists          8      16       64       64        128        256          512     1024
//   lengths     8000   1000-     300-    1500-      1500-      1500-        1500-     500-
//                       8000     4000    32768      32768      32768        32768     8192
//   1 CTA       64.4   63.6     34.9    247.9      247.3   (r)274.4     (r)342.5 (r)189.9
//   2           37.2   37.2     21.9    129.5   (r)144.1   (r)178.6     (r)350.4 (r)225.8
//   4           22.2   22.0     15.4     77.5    (r)96.3   (r)193.7     (r)380.8 (r)278.8
//   8           14.0   14.4  (r)18.9  (r)56.7   (r)114.2   (r)228.2     (r)451.1 (r)386.3
//   16          11.2   16.4  (r)40.6  (r)84.9   (r)168.6   (r)335.2     (r)651.0 (r)777.1
// The price: lists of equal length that a split makes more than fit (19 sequences of 16384:
// 142 us for 108). And keys are counted by the tables' capacity, as the lengths are on the
// device: 16 sequences of 500 tokens, 8 KV heads, take 10.7 us in tables of their length and
// 17.3 in tables of 32768 slots (one sequence of 2000 7.1 in both). The ranks cost every CTA a pass over the lengths and B comparisons for
// each of them, nothing where the lengths are alike: 128 sequences at most.
constexpr int MAX_SPLIT = 16;
int split_of(int64_t fit, int B, int64_t lists, int64_t keys) {
  int n = 1;
  while (n < MAX_SPLIT && lists * n * 2 <= (n == MAX_SPLIT / 2 ? num_sms() : fit) && keys / n > WARPS * 32) n *= 2;
  if (B > 1 && n < MAX_SPLIT && lists * n <= fit && keys / (2 * n) >= 1000) n *= 2;
  return n;
}

template <int D, bool FOLD>
dreams_status_t launch_rows(AttnParams P, cudaStream_t stream) {
  P.blocks = int32_t((int64_t(P.p.T_max) * P.p.G + RB - 1) / RB);
  const int64_t lists = int64_t(P.p.B) * P.p.Hkv * P.blocks;
  const int64_t fit = int64_t(Cfg8<D, FOLD>::PER_SM) * num_sms();
  P.p.nsplit = split_of(fit, P.p.B, lists, std::min<int64_t>(P.p.capacity, int64_t(P.p.window) - 1 + P.p.T_max + P.p.sinks));
  P.ranked = P.p.B > 1 && P.p.B <= MAX_RANKED && lists * P.p.nsplit > fit;
  return launch_lists<kv8_rows_kernel<D, FOLD>>(early_launch(), Cfg8<D, FOLD>::SMEM, lists, P.p.nsplit, stream, P);
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
  if (few <= (kv->D == 128 ? 2 : 4) * RB) return kv->D == 128 ? launch_rows<128, false>(P, s) : launch_rows<64, false>(P, s);
  return win::launch_tc8(P.p, P.c, kv->D, s);
}
