// kv8_attn.cu -- attention over a cache whose full pages are held in 8 bits.
#include <limits.h>
#include <math.h>

#include <algorithm>

#include "cache.cuh"
#include "kv8.cuh"

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
  const int64_t rows = int64_t(B) * T_max * Hq, blocks = (rows + 7) / 8;
  if (blocks > INT_MAX) return DREAMS_ERR_UNSUPPORTED;
  return launch(early_launch(), kv->D == 128 ? kv8_plain_kernel<128> : kv8_plain_kernel<64>, dim3(unsigned(blocks)), 256, 0, 1, stream, P);
}
