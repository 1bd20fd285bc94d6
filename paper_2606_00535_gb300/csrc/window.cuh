// window.cuh -- what the kernels of windowed attention share: the parameters, the
// key list of a block of query rows, and who sees what.
#pragma once
#include "common.cuh"
#include "tc.cuh"

namespace dreams {
namespace win {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;

struct WinParams {
  const __nv_bfloat16 *q;
  int64_t sb, st;  // strides of q in elements
  const __nv_bfloat16 *k, *v;
  __nv_bfloat16 *out;
  float *lse;
  const int32_t *table;  // nullptr: contiguous cache
  int32_t P, num_pages, capacity;
  const int32_t *parent;  // nullptr: causal
  const int32_t *q_len, *kv_len;
  int32_t B, T_max, Hq, Hkv, G;
  int32_t window, sinks;
  float scale_log2;
  int32_t nsplit;
  int32_t *status;
};

// The key list of a block of rows: slots 0 .. S1-1, then lo .. hi-1.
struct KeyList {
  int lo, S1, n;
  __device__ __forceinline__ int slot(int i) const { return i < S1 ? i : lo + (i - S1); }
};

__device__ __forceinline__ KeyList key_list(const WinParams &p, int L, int t_first, int t_last) {
  KeyList kl;
  const int p0 = L + (p.parent != nullptr ? 0 : t_first);  // no row of the block is before it
  kl.lo = ::max(0, p0 - p.window + 1);
  kl.S1 = ::min(p.sinks, kl.lo);
  kl.n = kl.S1 + (L + t_last + 1 - kl.lo);
  return kl;
}

// The new slots a tree node (t < q_len) sees, as a bit per node, and its depth: the
// walk from the node to the root over a checked parent array.
template <typename I>
__device__ __forceinline__ unsigned long long tree_row(const WinParams &p, const I *par, int L, int t, int &depth) {
  depth = -1;
  unsigned long long m = 0ull;
  for (int a = t; a >= 0; a = par[a], ++depth) m |= 1ull << a;
  if (depth >= p.window) {  // ancestors that the window has left behind
    int da = depth;
    for (int a = t; a >= 0; a = par[a], --da)
      if (depth - da >= p.window && int64_t(L) + da >= p.sinks) m &= ~(1ull << a);
  }
  return m;
}

__device__ __forceinline__ bool sees(const WinParams &p, int L, int off, unsigned long long anc, int slot) {
  const bool near = int64_t(L) + off - slot < p.window || slot < p.sinks;
  if (p.parent == nullptr) return near && slot <= L + off;
  return slot < L ? near : ((anc >> (slot - L)) & 1ull) != 0;
}

// Barriers of a cluster. Not the .aligned forms: a warp may come here from a loop that
// its lanes left at different turns.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }
__device__ __forceinline__ void cluster_sync() {
  __syncwarp();
  cluster_arrive();
  cluster_wait();
}
__device__ __forceinline__ uint32_t mapa(uint32_t addr, uint32_t cta) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(cta));
  return r;
}

// The checks of dreams_window_attention's arguments, and its parameters from them.
dreams_status_t window_args(const void *q, int64_t q_stride_b, int64_t q_stride_t, const dreams_kv_cache_t *kv, int32_t layer, const int32_t *parent,
                            const int32_t *q_len, const int32_t *kv_len, int32_t B, int32_t T_max, int32_t Hq, float scale, int32_t window,
                            int32_t sinks, void *out, float *lse, int32_t *status_word, WinParams &p);

// Blocks of 128 rows on the fifth-generation tensor cores (window_tc.cu).
dreams_status_t launch_tc(const WinParams &p, const dreams_kv_cache_t *kv, cudaStream_t stream);

}  // namespace win
}  // namespace dreams
