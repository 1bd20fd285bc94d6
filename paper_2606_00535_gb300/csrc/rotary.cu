// rotary.cu -- rotary positions: of any tensor (rope), and on the way of new rows
// into the cache (append).
//
// Pair (u, v) of a head's dimensions is turned by the angle a = 2 pi p f of its
// token's position p. f comes as a 64-bit fraction of a turn, so p f modulo one turn
// is one integer product, whose upper 32 bits, rounded to f32, give a within 2^-25 pi at
// any position (24 bits of up to half a turn); a position times an f32 frequency is off by
// 0.06 radians at a million. cos and sin are
// sincospif of it, f32 like the products, and the result is rounded once.
//
// Bound by HBM (each row read and written once), or by latency for few tokens. A
// block takes NT tokens of a sequence. Its threads first put their first rows' loads
// on their way, then work out the block's angles together, once for all heads, into
// shared memory; a thread then keeps the cosines and sines of the V pairs that it
// has in every head it goes over in registers.
// 3392 tokens of 32 heads of 128 dimensions, bf16: 11.3 us, 74% of the copy rate (from L2,
// which holds both sides, and with launch, angles and tail in it); rows of 16 chunks of up
// to 2048 tokens with 32 and 8 heads on their way into the cache: 94.6 us, 95% of it; one
// token of 28 heads 1.6 us, appended 2.3 us. Rows that are no whole 16-byte pieces go value by
// value: the same 3392 tokens with 24 of 96 dimensions turned 11.6 us, 32 of 96 9.6.
#include <limits.h>
#include <math.h>

#include <algorithm>

#include "cache.cuh"

namespace dreams {
namespace {

constexpr int THREADS = 256;
constexpr int BATCH = 4;  // heads of a thread on their way at once

struct RopeParams {
  const uint64_t *phase;
  const int32_t *axis;
  int32_t n;  // pairs
  float factor;
  const int32_t *positions;  // [axes, B, T]
  int32_t axes;
  const int32_t *start;   // [B]: of the tokens, or their slots
  const int32_t *parent;  // [B, T]
  const int32_t *n_new;   // append: rows per sequence; nullptr: T
  int32_t B, T;
  float sign;  // of the sines
  const void *x;  // the tensor, or Q
  int64_t xb, xt, xh;
  void *y;
  int64_t yb, yt, yh;
  int32_t H, D;  // heads of x
  // append
  const __nv_bfloat16 *k, *v;
  int64_t kb, kt, vb, vt;
  int32_t Hkv;
  Cache c;
  int32_t U, HL, NT;  // units of a head; heads side by side; tokens of a block
  Divisor per_token, per_head, pairs;  // HL * U, U, n
  int32_t *status;
};

// V elements of a row and their two halves' arithmetic in f32.
template <typename T, int V>
struct Piece;
template <>
struct Piece<__nv_bfloat16, 8> {
  uint4 w;
  __device__ __forceinline__ void load(const __nv_bfloat16 *p) { w = ld_stream(reinterpret_cast<const uint4 *>(p)); }
  __device__ __forceinline__ void store(__nv_bfloat16 *p) const { *reinterpret_cast<uint4 *>(p) = w; }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    const uint32_t a[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(a[i] << 16);
      f[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u);
    }
  }
  __device__ __forceinline__ void put(const float (&f)[8]) {
    w = make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
  }
};
template <>
struct Piece<float, 4> {
  uint4 w;
  __device__ __forceinline__ void load(const float *p) { w = ld_stream(reinterpret_cast<const uint4 *>(p)); }
  __device__ __forceinline__ void store(float *p) const { *reinterpret_cast<uint4 *>(p) = w; }
  __device__ __forceinline__ void get(float (&f)[4]) const {
    f[0] = __uint_as_float(w.x), f[1] = __uint_as_float(w.y), f[2] = __uint_as_float(w.z), f[3] = __uint_as_float(w.w);
  }
  __device__ __forceinline__ void put(const float (&f)[4]) {
    w = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
};
template <>
struct Piece<__nv_bfloat16, 1> {
  __nv_bfloat16 w;
  __device__ __forceinline__ void load(const __nv_bfloat16 *p) { w = *p; }
  __device__ __forceinline__ void store(__nv_bfloat16 *p) const { *p = w; }
  __device__ __forceinline__ void get(float (&f)[1]) const { f[0] = __bfloat162float(w); }
  __device__ __forceinline__ void put(const float (&f)[1]) { w = __float2bfloat16(f[0]); }
};
template <>
struct Piece<float, 1> {
  float w;
  __device__ __forceinline__ void load(const float *p) { w = *p; }
  __device__ __forceinline__ void store(float *p) const { *p = w; }
  __device__ __forceinline__ void get(float (&f)[1]) const { f[0] = w; }
  __device__ __forceinline__ void put(const float (&f)[1]) { w = f[0]; }
};

// A unit is two pieces of V dimensions of a head. HALF: piece d and its partner d + n
// where they are turned (n a multiple of V), else two neighbours; INTER: neighbours,
// whose pairs lie within them. V = 1 takes any n, D and alignment.
template <typename T, int V, bool INTER, bool APPEND>
__global__ void __launch_bounds__(THREADS) rope_kernel(const RopeParams p) {
  using P = Piece<T, V>;
  __shared__ float2 s_cs[2048];  // [token][V / 2][unit][2]; V = 1: [token][unit]
  __shared__ int s_par[64], s_pos[16];
  after_previous();
  const int tid = threadIdx.x, b = blockIdx.y;
  const int t0 = blockIdx.x * p.NT;
  int n = p.T, L = 0;
  if (APPEND) {
    n = p.n_new[b];
    L = p.start[b];
    if (n < 0 || n > p.T || L < 0 || int64_t(L) + n > p.c.capacity) {
      if (blockIdx.x == 0 && tid == 0) flag(p.status, DREAMS_DATA_BAD_KV_LEN);
      return;
    }
    if (t0 >= n) return;
    if (p.parent != nullptr) {
      int bad = 0;
      if (tid < n) {  // n <= 64
        const int q = p.parent[int64_t(b) * p.T + tid];
        s_par[tid] = q;
        bad = tid == 0 ? q != -1 : (q < 0 || q >= tid);
      }
      if (__syncthreads_or(bad)) {
        if (blockIdx.x == 0 && tid == 0) flag(p.status, DREAMS_DATA_BAD_PARENT);
        return;
      }
      if (tid < p.NT && t0 + tid < n) {
        int d = -1;
        for (int a = t0 + tid; a >= 0; a = s_par[a]) ++d;
        s_pos[tid] = L + d;
      }
      __syncthreads();
    }
  } else if (p.start != nullptr) {
    L = p.start[b];
  }
  const int tok = p.per_token.div(tid), in = tid - tok * int(p.per_token.d), hl = p.per_head.div(in), u = in - hl * p.U;
  const int t = t0 + tok;
  const bool mine = tok < p.NT && t < n;
  // the two pieces of this thread, and whether (HALF) they are a turned pair
  const bool turned = u * V < p.n;
  const int d0 = !INTER && turned ? u * V : 2 * u * V, d1 = !INTER && turned ? d0 + p.n : d0 + V;
  const int heads = APPEND ? p.H + 2 * p.Hkv : p.H;
  const T *x = static_cast<const T *>(p.x) + (mine ? b * p.xb + t * p.xt : 0);
  const T *k = nullptr, *v = nullptr;
  if (APPEND && mine) {
    k = reinterpret_cast<const T *>(p.k) + b * p.kb + t * p.kt;
    v = reinterpret_cast<const T *>(p.v) + b * p.vb + t * p.vt;
  }
  auto row = [&](int h) -> const T * {
    if (!APPEND) return x + h * p.xh;
    return h < p.H ? x + int64_t(h) * p.D : h < p.H + p.Hkv ? k + int64_t(h - p.H) * p.D : v + int64_t(h - p.H - p.Hkv) * p.D;
  };
  P a[BATCH], c[BATCH];
  auto load = [&](int h0) {
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const int h = h0 + i * p.HL;
      if (mine && h < heads) {
        const T *r = row(h);
        a[i].load(r + d0);
        c[i].load(r + d1);
      }
    }
  };
  load(hl);
  int64_t slot = -1;  // first element of the cache row
  if (APPEND && mine) {
    slot = slot16(p.c, b, L + t) * 8;
    if (slot < 0 && in == 0) flag(p.status, DREAMS_DATA_BAD_PAGE);
  }

  for (int i = tid; i < p.NT * p.n; i += THREADS) {
    const int j = p.pairs.div(i), q = i - j * p.n;
    if (t0 + j >= n) break;
    int64_t pos = int64_t(L) + t0 + j;
    if (APPEND && p.parent != nullptr) pos = s_pos[j];
    if (p.positions != nullptr) {
      int ax = p.axis != nullptr ? p.axis[q] : 0;
      if (ax < 0 || ax >= p.axes) {
        flag(p.status, DREAMS_DATA_BAD_INDEX);
        ax = 0;
      }
      pos = p.positions[(int64_t(ax) * p.B + b) * p.T + t0 + j];
    }
    const uint64_t turns = p.phase[q] * uint64_t(pos);
    float sn, cs;
    sincospif(float(int32_t(turns >> 32)) * 0x1p-31f, &sn, &cs);
    const int at = q / V, e = q % V;
    s_cs[V == 1 ? j * p.U + at : ((j * (V / 2) + e / 2) * p.U + at) * 2 + (e & 1)] = make_float2(cs * p.factor, sn * p.factor * p.sign);
  }
  __syncthreads();
  if (!mine) return;
  float cs[V], sn[V];
#pragma unroll
  for (int e = 0; e < V; e += V == 1 ? 1 : 2) {
    if constexpr (V == 1) {
      const float2 w = s_cs[tok * p.U + u];
      cs[0] = w.x, sn[0] = w.y;
    } else {
      const float4 w = *reinterpret_cast<const float4 *>(&s_cs[((tok * (V / 2) + e / 2) * p.U + u) * 2]);
      cs[e] = w.x, sn[e] = w.y, cs[e + 1] = w.z, sn[e + 1] = w.w;
    }
  }
  T *y = static_cast<T *>(p.y) + b * p.yb + t * p.yt;
  T *ck = nullptr, *cv = nullptr;
  if (APPEND && slot >= 0) {
    ck = reinterpret_cast<T *>(p.c.k) + slot;
    cv = reinterpret_cast<T *>(p.c.v) + slot;
  }
  for (int h0 = hl;;) {
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const int h = h0 + i * p.HL;
      if (h >= heads) break;
      const bool plain = APPEND && h >= p.H + p.Hkv;
      if (!plain && (INTER || turned)) {
        float f[V], g[V];
        a[i].get(f);
        c[i].get(g);
        if constexpr (INTER) {
#pragma unroll
          for (int e = 0; e < V / 2; ++e) {
            if (u * V + e < p.n) {
              const float r = f[2 * e], s = f[2 * e + 1];
              f[2 * e] = r * cs[e] - s * sn[e];
              f[2 * e + 1] = s * cs[e] + r * sn[e];
            }
            if (u * V + V / 2 + e < p.n) {
              const float r = g[2 * e], s = g[2 * e + 1];
              g[2 * e] = r * cs[V / 2 + e] - s * sn[V / 2 + e];
              g[2 * e + 1] = s * cs[V / 2 + e] + r * sn[V / 2 + e];
            }
          }
          if constexpr (V == 1) {  // the two pieces are the pair
            if (turned) {
              const float r = f[0], s = g[0];
              f[0] = r * cs[0] - s * sn[0];
              g[0] = s * cs[0] + r * sn[0];
            }
          }
        } else {
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const float r = f[e], s = g[e];
            f[e] = r * cs[e] - s * sn[e];
            g[e] = s * cs[e] + r * sn[e];
          }
        }
        a[i].put(f);
        c[i].put(g);
      }
      T *to;
      if (!APPEND) {
        to = y + h * p.yh;
      } else if (h < p.H) {
        to = y + int64_t(h) * p.D;
      } else {
        if (slot < 0) break;
        to = h < p.H + p.Hkv ? ck + int64_t(h - p.H) * p.D : cv + int64_t(h - p.H - p.Hkv) * p.D;
      }
      a[i].store(to + d0);
      c[i].store(to + d1);
    }
    h0 += BATCH * p.HL;
    if (h0 >= heads) break;
    load(h0);
  }
}

// ------------------------------------------------------------------ host side
bool rotary_ok(const dreams_rotary_t *r, int D) {
  return r != nullptr && r->phase != nullptr && (reinterpret_cast<uintptr_t>(r->phase) & 7u) == 0 && aligned4(r->axis) && r->n_pairs >= 1 &&
         r->n_pairs <= D / 2 && (r->layout == DREAMS_ROPE_HALF || r->layout == DREAMS_ROPE_INTERLEAVED) && isfinite(r->factor);
}

// Every dimension is stepped over by more than what lies inside it.
bool no_overlap(const int64_t *stride, const int32_t *size, int D) {
  int order[3] = {0, 1, 2};
  std::sort(order, order + 3, [&](int i, int j) { return stride[i] < stride[j]; });
  int64_t extent = D;
  for (int i : order) {
    if (size[i] == 1) continue;
    if (stride[i] < extent) return false;
    extent = stride[i] * int64_t(size[i] - 1) + extent;
  }
  return true;
}

template <typename T, int V>
dreams_status_t launch_rope(RopeParams &p, bool inter, bool append, dreams_stream_t stream) {
  const int heads = append ? p.H + 2 * p.Hkv : p.H;
  p.U = p.D / (2 * V);
  // Threads of a token: a quarter of a block where there are tokens for all SMs, a
  // whole one where not.
  const int64_t blocks4 = int64_t(p.B) * ((p.T + 3) / 4);
  const int want = blocks4 >= num_sms() ? THREADS / 4 : THREADS;
  p.HL = std::max(1, std::min(heads, want / p.U));
  p.NT = std::max(1, std::min({p.T, 16, blocks4 >= num_sms() ? THREADS / (p.U * p.HL) : 1}));
  p.per_token = Divisor::of(int64_t(p.HL) * p.U);
  p.per_head = Divisor::of(p.U);
  p.pairs = Divisor::of(p.n);
  const dim3 grid(unsigned((p.T + p.NT - 1) / p.NT), unsigned(p.B));
  if constexpr (sizeof(T) == 2) {
    if (append) return launch(early_launch(), inter ? rope_kernel<T, V, true, true> : rope_kernel<T, V, false, true>, grid, THREADS, 0, 1, stream, p);
  }
  return launch(early_launch(), inter ? rope_kernel<T, V, true, false> : rope_kernel<T, V, false, false>, grid, THREADS, 0, 1, stream, p);
}

}  // namespace
}  // namespace dreams

using namespace dreams;

extern "C" dreams_status_t dreams_rope(const void *x, int64_t x_stride_b, int64_t x_stride_t, int64_t x_stride_h, void *out, int64_t out_stride_b,
                                       int64_t out_stride_t, int64_t out_stride_h, dreams_dtype_t dtype, int32_t B, int32_t T, int32_t H, int32_t D, const dreams_rotary_t *rotary, const int32_t *positions,
                                       int32_t n_axes, const int32_t *start, int32_t transpose, int32_t *status_word, dreams_stream_t stream) {
  if (x == nullptr || out == nullptr || (dtype != DREAMS_F32 && dtype != DREAMS_BF16) || B < 1 ||
      B > 65535 || T < 1 || T > (1 << 30) || H < 1 || H > (1 << 20) || D < 2 || D % 2 != 0 || D > 512 || !rotary_ok(rotary, D) || n_axes < 1 ||
      n_axes > 4 || !aligned4(positions) || !aligned4(start) || (positions != nullptr && start != nullptr) || (positions == nullptr && n_axes != 1))
    return DREAMS_ERR_INVALID_ARG;
  const int es = dtype == DREAMS_F32 ? 4 : 2;
  if (reinterpret_cast<uintptr_t>(x) % es != 0 || reinterpret_cast<uintptr_t>(out) % es != 0) return DREAMS_ERR_INVALID_ARG;
  const int32_t size[3] = {B, T, H};
  const int64_t x_stride[3] = {x_stride_b, x_stride_t, x_stride_h}, out_stride[3] = {out_stride_b, out_stride_t, out_stride_h};
  int64_t xs[3], ys[3];
  uint64_t odd = (reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(out)) & 15u;
  for (int i = 0; i < 3; ++i) {  // (the stride of a dimension of one says nothing)
    xs[i] = size[i] > 1 ? x_stride[i] : 0;
    ys[i] = size[i] > 1 ? out_stride[i] : 0;
    if (xs[i] < 0 || ys[i] < 0 || xs[i] >= (int64_t(1) << 38) || ys[i] >= (int64_t(1) << 38)) return DREAMS_ERR_INVALID_ARG;
    if (x == out && xs[i] != ys[i]) return DREAMS_ERR_INVALID_ARG;
    odd |= uint64_t(xs[i] * es | ys[i] * es) & 15u;
  }
  if (!no_overlap(ys, size, D)) return DREAMS_ERR_INVALID_ARG;
  RopeParams p{};
  p.phase = rotary->phase;
  p.axis = rotary->axis;
  p.n = rotary->n_pairs;
  p.factor = rotary->factor;
  p.positions = positions;
  p.axes = n_axes;
  p.start = start;
  p.B = B;
  p.T = T;
  p.sign = transpose != 0 ? -1.f : 1.f;
  p.x = x;
  p.xb = xs[0], p.xt = xs[1], p.xh = xs[2];
  p.y = out;
  p.yb = ys[0], p.yt = ys[1], p.yh = ys[2];
  p.H = H;
  p.D = D;
  p.status = status_word;
  const bool inter = rotary->layout == DREAMS_ROPE_INTERLEAVED;
  const int V = 16 / es;
  const bool wide = odd == 0 && D % (2 * V) == 0 && (inter || p.n % V == 0);
  if (dtype == DREAMS_F32) return wide ? launch_rope<float, 4>(p, inter, false, stream) : launch_rope<float, 1>(p, inter, false, stream);
  return wide ? launch_rope<__nv_bfloat16, 8>(p, inter, false, stream) : launch_rope<__nv_bfloat16, 1>(p, inter, false, stream);
}

extern "C" dreams_status_t dreams_kv_append_rope(const dreams_kv_cache_t *kv, int32_t layer, const void *q, int64_t q_stride_b, int64_t q_stride_t,
                                                 void *q_out, int32_t Hq, const void *k_new, int64_t k_stride_b, int64_t k_stride_t,
                                                 const void *v_new, int64_t v_stride_b, int64_t v_stride_t, const dreams_rotary_t *rotary, const int32_t *positions, int32_t n_axes, const int32_t *parent,
                                                 const int32_t *kv_len, const int32_t *n_new, int32_t B, int32_t T_max, int32_t *status_word,
                                                 dreams_stream_t stream) {
  Cache c;
  if (!cache_ok(kv, c) || layer < 0 || layer >= kv->n_layers || k_new == nullptr || v_new == nullptr ||
      kv_len == nullptr || n_new == nullptr || B < 1 || B > 65535 || T_max < 1 || T_max > (parent != nullptr ? 64 : 1 << 20) || !aligned16(k_new) ||
      !aligned16(v_new) || !aligned4(kv_len) || !aligned4(n_new) || !aligned4(parent) || !aligned4(positions) || n_axes < 1 || n_axes > 4 ||
      (positions != nullptr && parent != nullptr) || (positions == nullptr && n_axes != 1) || kv->D > 512 || !rotary_ok(rotary, kv->D))
    return DREAMS_ERR_INVALID_ARG;
  if (q == nullptr ? (q_out != nullptr || Hq != 0)
                   : (q_out == nullptr || Hq < 1 || Hq > (1 << 20) || !aligned16(q) || !aligned16(q_out)))
    return DREAMS_ERR_INVALID_ARG;
  const int64_t D = kv->D;
  int64_t s[3][2] = {};
  const int64_t given[3][2] = {{q_stride_b, q_stride_t}, {k_stride_b, k_stride_t}, {v_stride_b, v_stride_t}};
  for (int i = q == nullptr ? 1 : 0; i < 3; ++i) {
    const int64_t row = (i == 0 ? Hq : kv->Hkv) * D;
    s[i][1] = T_max == 1 ? row : given[i][1];
    s[i][0] = B == 1 ? s[i][1] : given[i][0];
    for (const int64_t x : s[i])
      if (x < row || x % 8 != 0 || x >= (int64_t(1) << 38)) return DREAMS_ERR_INVALID_ARG;
  }
  if (q != nullptr && q == q_out && ((T_max > 1 && s[0][1] != Hq * D) || (B > 1 && s[0][0] != T_max * int64_t(Hq) * D))) return DREAMS_ERR_INVALID_ARG;
  c.k += layer * c.layer16;
  c.v += layer * c.layer16;
  RopeParams p{};
  p.phase = rotary->phase;
  p.axis = rotary->axis;
  p.n = rotary->n_pairs;
  p.factor = rotary->factor;
  p.positions = positions;
  p.axes = n_axes;
  p.start = kv_len;
  p.parent = parent;
  p.n_new = n_new;
  p.B = B;
  p.T = T_max;
  p.sign = 1.f;
  p.x = q;
  p.xb = s[0][0], p.xt = s[0][1];
  p.y = q_out;
  p.yb = T_max * int64_t(Hq) * D, p.yt = Hq * D;
  p.H = Hq;
  p.D = kv->D;
  p.k = static_cast<const __nv_bfloat16 *>(k_new);
  p.v = static_cast<const __nv_bfloat16 *>(v_new);
  p.kb = s[1][0], p.kt = s[1][1], p.vb = s[2][0], p.vt = s[2][1];
  p.Hkv = kv->Hkv;
  p.c = c;
  p.status = status_word;
  const bool inter = rotary->layout == DREAMS_ROPE_INTERLEAVED;
  if (D % 16 == 0 && (inter || p.n % 8 == 0)) return launch_rope<__nv_bfloat16, 8>(p, inter, true, stream);
  return launch_rope<__nv_bfloat16, 1>(p, inter, true, stream);
}
