// cache.cuh -- what the kernels that move rows of the KV cache share: the cache as
// 16-byte columns, its check, and their launch.
#pragma once
#include "common.cuh"

namespace dreams {

constexpr int PAGE = 64;

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
  const int pg = c.table[int64_t(b) * c.P + (s >> 6)];
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

// ------------------------------------------------------------------ host side
inline bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

inline bool cache_ok(const dreams_kv_cache_t *kv, Cache &c) {
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

// (a head dim that a call does not serve is its own affair)
inline bool kv8_ok(const dreams_kv8_cache_t *c) {
  return c != nullptr && c->k != nullptr && c->v != nullptr && c->exps != nullptr && c->page_table != nullptr && c->n_layers >= 1 && c->Hkv >= 1 &&
         c->Hkv <= 65535 && c->D >= 1 && c->layer_stride >= 0 && c->layer_stride % 16 == 0 && aligned16(c->k) && aligned16(c->v) && aligned4(c->exps) &&
         aligned4(c->page_table) && c->pages_per_seq >= 1 && c->num_pages >= 1 && int64_t(c->pages_per_seq) * PAGE <= INT_MAX;
}

template <typename... Params, typename... Args>
dreams_status_t launch(cudaLaunchAttribute first, void (*kernel)(Params...), dim3 grid, int threads, size_t smem, int cluster, dreams_stream_t stream,
                       const Args &...args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(unsigned(threads));
  cfg.dynamicSmemBytes = smem;
  cfg.stream = reinterpret_cast<cudaStream_t>(stream);
  cudaLaunchAttribute attr[2] = {first};
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = unsigned(cluster);
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, Params(args)...);
  if (e != cudaSuccess) {
    set_last_cuda_error(e);
    return DREAMS_ERR_CUDA;
  }
  return check_launch();
}

}  // namespace dreams
