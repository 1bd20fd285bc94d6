// kv8.cu -- full pages of the cache put into 8 bits.
//
// Of each page and head, K and V apart, the power of two is the smallest with
// max |x| <= 448 2^e (448 = 1.75 2^8 is e4m3's largest value), read off the exponent and
// mantissa of the largest magnitude, and a code is x 2^-e rounded to nearest even. A
// power of two keeps e4m3's relative precision, and codes times powers are exact in
// bf16, so the attention works on the very values that are stored.
//
// Bound by HBM: two bytes of a value read, one written. A block takes a page of a
// layer's head, K and V, 64 rows of each in registers between the maximum and the
// rounding. Blocks are persistent, as which pages there are is known on the device
// alone: each counts the pages of 256 sequences at a time by a prefix sum and walks
// over (page, layer, head), heads side by side, so that neighbours read neighbouring
// parts of the same rows. 3392 tokens of 32 layers of 32 heads: 425 us, 94% of the copy rate;
// one page of 8 layers of 8 heads for each of 16 sequences 11.1 us, of which 7.6 are the bytes.
#include <limits.h>

#include <algorithm>

#include "cache.cuh"
#include "kv8.cuh"

namespace dreams {
namespace {

constexpr int THREADS = 256;
// Blocks of an SM, all of which run: 3392 tokens of 32 heads and layers, head dim 128, take
// 425 us with 4, 471 with 3 and 579 with 6 (spills); 16 x 1000 to 3000 of 8 heads and layers,
// head dim 64, 149 with 6 and 166 with 4.
template <int D>
constexpr int RESIDENT = D == 64 ? 6 : 4;

struct QuantParams {
  Cache c;
  uint8_t *k8, *v8;
  uint32_t *exps;
  int64_t stride8;  // bytes of a layer
  const int32_t *table8;
  int32_t P8, num_pages8;
  int32_t B, Hkv, n_layers;
  const int32_t *begin, *end;
  int32_t *new_len8;
  int32_t *status;
};

__device__ __forceinline__ int page16(const QuantParams &p, int b, int e) {
  if (p.c.table == nullptr) return 0;
  const int pg = p.c.table[int64_t(b) * p.c.P + e];
  return pg < p.c.num_pages ? pg : -1;
}
__device__ __forceinline__ int page8(const QuantParams &p, int b, int e) {
  const int pg = p.table8[int64_t(b) * p.P8 + e];
  return pg < p.num_pages8 ? pg : -1;
}

// The power for a largest magnitude of these bf16 bits.
__device__ __forceinline__ int power_for(uint32_t bits) {
  if (bits >= 0x7f80u) return DREAMS_KV8_NOT_FINITE;
  return ::min(::max(int(bits >> 7) - 135 + int((bits & 0x7fu) > 96u), EXP_MIN), EXP_MAX);
}

// Two bf16 as codes, the first in the low byte.
__device__ __forceinline__ uint32_t to_codes(uint32_t w, float scale) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(__uint_as_float(w & 0xffff0000u) * scale), "f"(__uint_as_float(w << 16) * scale));
  return r;
}

template <int D>
__global__ void __launch_bounds__(THREADS, RESIDENT<D>) kv_quantize_kernel(const QuantParams p) {
  constexpr int COLS = D / 8, ROWS = THREADS / COLS, N = PAGE / ROWS;  // 16-byte columns; rows of a pass; passes
  __shared__ int s_first[THREADS + 1], s_warp[THREADS / 32];
  __shared__ uint32_t s_max[2][THREADS / 32];  // K's in the low half, V's in the high one
  after_previous();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int row = tid / COLS, col = tid % COLS;
  int turn = 0;
  for (int b0 = 0; b0 < p.B; b0 += THREADS) {
    // the pages of these sequences
    const int b = b0 + tid;
    int n = 0;
    if (b < p.B) {
      const int from = p.begin[b], to = p.end[b];
      const bool bad = from < 0 || (from & 63) != 0 || to < from || to > p.c.capacity || int64_t(to >> 6) > p.P8;
      if (bad) {
        if (blockIdx.x == 0) {
          flag(p.status, DREAMS_DATA_BAD_KV_LEN);
          p.new_len8[b] = from;
        }
      } else {
        n = (to >> 6) - (from >> 6);
        if (n == 0 && blockIdx.x == 0) p.new_len8[b] = from;
      }
    }
    int sum = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int z = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += z;
    }
    if (lane == 31) s_warp[warp] = sum;
    __syncthreads();
    for (int w = 0; w < warp; ++w) sum += s_warp[w];
    s_first[tid + 1] = sum;
    if (tid == 0) s_first[0] = 0;
    __syncthreads();
    const int pages = s_first[THREADS];
    // the new lengths: a warp walks a sequence's entries up to the first that is missing
    for (int i = int(blockIdx.x) + warp * int(gridDim.x); i < THREADS && b0 + i < p.B; i += int(gridDim.x) * (THREADS / 32)) {
      const int count = s_first[i + 1] - s_first[i];
      if (count == 0) continue;
      const int e0 = p.begin[b0 + i] >> 6;
      int done = 0;
      for (; done < count; done += 32) {
        const int e = e0 + done + lane;
        const unsigned missing = __ballot_sync(0xffffffffu, done + lane < count && (page16(p, b0 + i, e) < 0 || page8(p, b0 + i, e) < 0));
        if (missing != 0) {
          done += __ffs(int(missing)) - 1;
          break;
        }
      }
      if (lane == 0) p.new_len8[b0 + i] = (e0 + ::min(done, count)) << 6;
    }
    const int64_t items = int64_t(pages) * p.n_layers * p.Hkv;
    for (int64_t x = blockIdx.x; x < items; x += gridDim.x) {
      const int64_t y = x / p.Hkv;
      const int g = int(x - y * p.Hkv), pi = int(y / p.n_layers), layer = int(y - int64_t(pi) * p.n_layers);
      int lo = 0, hi = THREADS;  // the sequence: the last i with first[i] <= pi
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        (s_first[mid] <= pi ? lo : hi) = mid;
      }
      const int e = (p.begin[b0 + lo] >> 6) + pi - s_first[lo];
      const int pg = page16(p, b0 + lo, e), pg8 = page8(p, b0 + lo, e);
      if (pg < 0 || pg8 < 0) {
        if (tid == 0 && g == 0 && layer == 0) flag(p.status, DREAMS_DATA_BAD_PAGE);
        continue;
      }
      const int64_t slot = p.c.table == nullptr ? int64_t(b0 + lo) * p.c.capacity + e * PAGE : int64_t(pg) * PAGE;
      const int64_t at = layer * p.c.layer16 + (slot + row) * p.c.row16 + g * COLS + col;
      uint4 kk[N], vv[N];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        kk[i] = ld_stream(p.c.k + at + int64_t(i) * ROWS * p.c.row16);
        vv[i] = ld_stream(p.c.v + at + int64_t(i) * ROWS * p.c.row16);
      }
      uint32_t mk = 0, mv = 0;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        mk = __vmaxu2(mk, __vmaxu2(__vmaxu2(kk[i].x & 0x7fff7fffu, kk[i].y & 0x7fff7fffu), __vmaxu2(kk[i].z & 0x7fff7fffu, kk[i].w & 0x7fff7fffu)));
        mv = __vmaxu2(mv, __vmaxu2(__vmaxu2(vv[i].x & 0x7fff7fffu, vv[i].y & 0x7fff7fffu), __vmaxu2(vv[i].z & 0x7fff7fffu, vv[i].w & 0x7fff7fffu)));
      }
      mk = __reduce_max_sync(0xffffffffu, ::max(mk & 0xffffu, mk >> 16));
      mv = __reduce_max_sync(0xffffffffu, ::max(mv & 0xffffu, mv >> 16));
      if (lane == 0) s_max[turn][warp] = mk | mv << 16;
      __syncthreads();
      uint32_t most = 0;
#pragma unroll
      for (int w = 0; w < THREADS / 32; ++w) most = __vmaxu2(most, s_max[turn][w]);
      turn ^= 1;  // (the next item's barrier lies between this read and the next write here)
      const int ek = power_for(most & 0xffffu), ev = power_for(most >> 16);
      const float fk = power(ek == DREAMS_KV8_NOT_FINITE ? 0 : -ek), fv = power(ev == DREAMS_KV8_NOT_FINITE ? 0 : -ev);
      const int64_t to = layer * p.stride8 + ((int64_t(pg8) * PAGE + row) * p.Hkv + g) * D + col * 8;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int64_t o = to + int64_t(i) * ROWS * p.Hkv * D;
        *reinterpret_cast<uint2 *>(p.k8 + o) = make_uint2(to_codes(kk[i].x, fk) | to_codes(kk[i].y, fk) << 16, to_codes(kk[i].z, fk) | to_codes(kk[i].w, fk) << 16);
        *reinterpret_cast<uint2 *>(p.v8 + o) = make_uint2(to_codes(vv[i].x, fv) | to_codes(vv[i].y, fv) << 16, to_codes(vv[i].z, fv) | to_codes(vv[i].w, fv) << 16);
      }
      if (tid == 0) p.exps[(int64_t(layer) * p.num_pages8 + pg8) * p.Hkv + g] = (uint32_t(ek) & 0xffffu) | uint32_t(ev) << 16;
    }
    __syncthreads();  // s_first is read no more
  }
}

// Blocks read begin and end while others write new lengths: read twice, an overwritten
// begin would lead behind the table's row.
bool apart(const int32_t *x, const int32_t *y, int n) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(x), b = reinterpret_cast<uintptr_t>(y), bytes = uintptr_t(n) * 4;
  return a + bytes <= b || b + bytes <= a;
}

}  // namespace
}  // namespace dreams

using namespace dreams;

extern "C" dreams_status_t dreams_kv_quantize(const dreams_kv_cache_t *kv, const dreams_kv8_cache_t *kv8, int32_t B, const int32_t *begin,
                                              const int32_t *end, int32_t *new_len8, int32_t *status_word, dreams_stream_t stream) {
  Cache c;
  if (!cache_ok(kv, c) || !kv8_ok(kv8) || B < 1 || B > 65535 || begin == nullptr || end == nullptr || new_len8 == nullptr || !aligned4(begin) ||
      !aligned4(end) || !aligned4(new_len8) || !apart(new_len8, begin, B) || !apart(new_len8, end, B) || kv8->n_layers != kv->n_layers || kv8->Hkv != kv->Hkv ||
      kv8->D != kv->D)
    return DREAMS_ERR_INVALID_ARG;
  // (a block counts the pages of THREADS sequences in 32 bits)
  if ((kv->D != 64 && kv->D != 128) || kv8->pages_per_seq > INT_MAX / THREADS) return DREAMS_ERR_UNSUPPORTED;
  QuantParams p{};
  p.c = c;
  p.k8 = static_cast<uint8_t *>(kv8->k);
  p.v8 = static_cast<uint8_t *>(kv8->v);
  p.exps = reinterpret_cast<uint32_t *>(kv8->exps);
  p.stride8 = kv8->layer_stride;
  p.table8 = kv8->page_table;
  p.P8 = kv8->pages_per_seq;
  p.num_pages8 = kv8->num_pages;
  p.B = B;
  p.Hkv = kv->Hkv;
  p.n_layers = kv->n_layers;
  p.begin = begin;
  p.end = end;
  p.new_len8 = new_len8;
  p.status = status_word;
  const int64_t most = int64_t(B) * std::min<int64_t>(kv8->pages_per_seq, kv->capacity / PAGE) * kv->n_layers * kv->Hkv;
  const dim3 grid(unsigned(std::max<int64_t>(1, std::min<int64_t>(most, int64_t(num_sms()) * (kv->D == 128 ? RESIDENT<128> : RESIDENT<64>)))));
  return launch(early_launch(), kv->D == 128 ? kv_quantize_kernel<128> : kv_quantize_kernel<64>, grid, THREADS, 0, 1, stream, p);
}
