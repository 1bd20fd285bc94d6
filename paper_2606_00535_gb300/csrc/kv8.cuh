// kv8.cuh -- full pages of the cache in 8 bits: e4m3 codes and a power of two per page,
// head, and K or V.
#pragma once
#include "common.cuh"
#include "window.cuh"

namespace dreams {

// Powers that are used. A code, 2^-9 to 448, times its power is a normal and finite bf16 at
// both ends, as the kernel for blocks makes it. A page of smaller values loses those below
// half of 2^-9 2^EXP_MIN; larger ones become 448 2^EXP_MAX.
constexpr int EXP_MIN = -96, EXP_MAX = 119;

struct Kv8 {
  const uint8_t *k, *v;  // one layer's
  const uint32_t *exps;  // [page][head]: K's in the low half, V's in the high one
  const int32_t *table;
  int32_t P, num_pages;
  const int32_t *len8;
};

__device__ __forceinline__ bool len8_bad(const Kv8 &c, int len8, int L) {
  return len8 < 0 || (len8 & 63) != 0 || len8 > L || int64_t(len8) > int64_t(c.P) * 64;
}

// 2^e; NaN for DREAMS_KV8_NOT_FINITE.
__device__ __forceinline__ float power(int e) {
  if (e == DREAMS_KV8_NOT_FINITE) return __uint_as_float(0x7fffffffu);
  return e >= -126 ? __uint_as_float(uint32_t(::min(e, 127) + 127) << 23) : 0.f;
}
__device__ __forceinline__ int k_exp(uint32_t w) { return int(int16_t(w & 0xffffu)); }
__device__ __forceinline__ int v_exp(uint32_t w) { return int(int16_t(w >> 16)); }

// Two codes as bf16 times 2^-120: a code's sign goes to bit 15, its four exponent and
// three mantissa bits to 10 .. 4, so the value is short of e4m3's by the difference of
// the formats' biases, 127 - 7, subnormals too. SEL picks the bytes, each followed by
// its sign spread over a byte.
template <uint32_t SEL>
__device__ __forceinline__ uint32_t codes_x2(uint32_t w) {
  uint32_t y;
  asm("prmt.b32 %0, %1, 0, %2;" : "=r"(y) : "r"(w), "n"(SEL));
  return (y << 4) & 0x87f087f0u;
}
constexpr uint32_t sel_of(int i, int j) { return uint32_t((8 | j) << 12 | j << 8 | (8 | i) << 4 | i); }

__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}

// One code's value.
__device__ __forceinline__ float code_value(uint32_t code) {
  const uint32_t u = (code & 0x80u) << 24 | (code & 0x7fu) << 20;
  return __uint_as_float(u) * 0x1p120f;
}

namespace win {
// Blocks of 128 rows over a cache in 8 bits (window_tc.cu).
dreams_status_t launch_tc8(const WinParams &p, const Kv8 &c, int D, cudaStream_t stream);
}  // namespace win

}  // namespace dreams
