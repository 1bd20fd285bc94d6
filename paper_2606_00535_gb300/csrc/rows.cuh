// rows.cuh -- attention for at most 16 query rows of a KV head: what its kernels share.
// Rows, the tensor instructions for 16 of them, and the join of the parts of a key list
// that warps and the CTAs of a cluster have streamed.
#pragma once
#include <limits.h>

#include <atomic>

#include "window.cuh"

namespace dreams {
namespace win {

constexpr int RB = 16;    // query rows of a CTA
constexpr int WARPS = 4;

__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// What a row of the block is: its position, and for a tree its visible new slots.
struct RowInfo {
  int off;                 // position - L; -1: no row
  unsigned long long anc;  // tree: bit a = sees slot L + a
};

struct RowsShared {
  int par[64];
  RowInfo row[RB];
  float2 ml[WARPS][RB];    // the warps' maxima and sums
  float2 part[16][RB];     // those of a list's parts
};

// The queries of a sequence and KV head, from row `first` on; false (flagged by
// `report`): a bad tree.
__device__ __forceinline__ bool load_rows(const WinParams &p, RowsShared &sh, int b, int L, int T, bool report, int first = 0) {
  const int tid = threadIdx.x;
  __syncthreads();  // the last part's readers are done
  if (p.parent != nullptr) {
    int bad = 0;
    for (int i = tid; i < T; i += 32 * WARPS) {
      const int par = p.parent[int64_t(b) * p.T_max + i];
      sh.par[i] = par;
      bad |= i == 0 ? par != -1 : (par < 0 || par >= i);
    }
    if (__syncthreads_or(bad)) {
      if (report && tid == 0) flag(p.status, DREAMS_DATA_BAD_PARENT);
      return false;
    }
  }
  if (tid < RB) {
    const int t = (first + tid) / p.G;
    RowInfo r{-1, 0ull};
    if (t < T) {
      r.off = t;
      if (p.parent != nullptr) r.anc = tree_row(p, sh.par, L, t, r.off);
    }
    sh.row[tid] = r;
  }
  __syncthreads();
  return true;
}

// Parts joined by log-sum-exp: sum of 2^(m_i - M) (l_i, o_i) over n parts, in order.
template <int UNROLL, typename ML, typename O>
__device__ __forceinline__ float4 join(int n, ML ml_of, O o_of, float &M, float &Z) {
  M = -INFINITY;
#pragma unroll UNROLL
  for (int i = 0; i < n; ++i) M = fmaxf(M, ml_of(i).x);
  Z = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll UNROLL
  for (int i = 0; i < n; ++i) {
    const float2 ml = ml_of(i);
    const float4 o = o_of(i);
    const bool some = ml.y != 0.f;  // (a NaN sum goes through; without keys o may hold anything)
    const float c = some ? tc::ex2(ml.x - M) : 0.f;
    Z += some ? c * ml.y : 0.f;
    acc.x += some ? c * o.x : 0.f;
    acc.y += some ? c * o.y : 0.f;
    acc.z += some ? c * o.z : 0.f;
    acc.w += some ? c * o.w : 0.f;
  }
  return acc;
}

// Unit u of the rows: row u / (D / 4), four columns.
template <int D>
__device__ __forceinline__ float4 join_warps(const RowsShared &sh, const uint8_t *smem, int u, float &M, float &Z) {
  const float *so = reinterpret_cast<const float *>(smem);
  const int r = u / (D / 4), d = (u % (D / 4)) * 4;
  return join<WARPS>(
      WARPS, [&](int w) { return sh.ml[w][r]; },
      [&](int w) { return *reinterpret_cast<const float4 *>(so + (w * RB + r) * D + d); }, M, Z);
}

template <int D>
__device__ __forceinline__ void emit(const WinParams &p, int b, int g, int u, float4 v, float M, float Z, int first) {
  const int r = first + u / (D / 4), d = (u % (D / 4)) * 4, t = r / p.G;
  const int64_t row = (int64_t(b) * p.T_max + t) * p.Hq + g * p.G + (r - t * p.G);
  const float inv = __frcp_rn(Z);
  *reinterpret_cast<uint2 *>(p.out + row * D + d) = make_uint2(pack_bf16x2(v.x * inv, v.y * inv), pack_bf16x2(v.z * inv, v.w * inv));
  if (d == 0 && p.lse != nullptr) p.lse[row] = (M + log2f(Z)) * LN2;
}

// Joins the warps' parts, which lie in `smem` as [warp][row][D] f32, and those of a
// cluster's CTAs, and writes the rows out. Behind ring_bytes there is room for RB * D * 4
// bytes that the CTAs push.
template <int D>
__device__ __forceinline__ void finish_rows(const WinParams &p, RowsShared &sh, uint8_t *smem, uint32_t ring_bytes, int b, int g, int T, int split,
                                            int first = 0) {
  const int tid = threadIdx.x;
  const int units = ::min(RB, T * p.G - first) * (D / 4);
  if (p.nsplit == 1) {
    for (int u = tid; u < units; u += 32 * WARPS) {
      float M, Z;
      const float4 v = join_warps<D>(sh, smem, u, M, Z);
      emit<D>(p, b, g, u, v, M, Z, first);
    }
    return;
  }
  // Unit u goes to CTA u % nsplit, place u / nsplit of this CTA's row there.
  cluster_wait();
  const uint32_t box = smem_u32(smem) + ring_bytes, part = smem_u32(&sh.part[0][0]);
  const int room = RB * (D / 4) / p.nsplit;  // units of a CTA
  for (int u = tid; u < units; u += 32 * WARPS) {
    float M, Z;
    const float4 v = join_warps<D>(sh, smem, u, M, Z);
    const int to = u % p.nsplit;
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1,%2,%3,%4};" ::"r"(mapa(box + (split * room + u / p.nsplit) * 16, to)), "f"(v.x),
                 "f"(v.y), "f"(v.z), "f"(v.w)
                 : "memory");
    if (u % (D / 4) < p.nsplit)  // the row's (M, Z) to every CTA, one thread each
      asm volatile("st.shared::cluster.v2.f32 [%0], {%1,%2};" ::"r"(mapa(part + (split * RB + u / (D / 4)) * 8, u % (D / 4))), "f"(M), "f"(Z)
                   : "memory");
  }
  cluster_sync();
  const float4 *in = reinterpret_cast<const float4 *>(smem + ring_bytes);
  for (int u = split + p.nsplit * tid; u < units; u += p.nsplit * 32 * WARPS) {
    float M, Z;
    const float4 v = join<4>(
        p.nsplit, [&](int c) { return sh.part[c][u / (D / 4)]; }, [&](int c) { return in[c * room + u / p.nsplit]; }, M, Z);
    emit<D>(p, b, g, u, v, M, Z, first);
  }
}

// ------------------------------------------------------------------ host side
// One CTA, or a cluster of nsplit, to each of `lists` key lists.
template <auto KERNEL, typename Params>
dreams_status_t launch_lists(cudaLaunchAttribute first, int smem, int64_t lists, int nsplit, cudaStream_t stream, Params p) {
  const void *kernel = reinterpret_cast<const void *>(KERNEL);
  const dreams_status_t st = ensure_max_dynamic_smem(kernel, smem);
  if (st != DREAMS_OK) return st;
  if (nsplit > 8) {
    // clusters of 16 have to be asked for, once per device; without a lock, as single tokens'
    // calls are bound by the host
    static std::atomic<uint64_t> wide{0};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess && (dev >= 64 || !((wide.load() >> dev) & 1u))) {
      e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
      if (e == cudaSuccess && dev < 64) wide.fetch_or(uint64_t(1) << dev);
    }
    if (e != cudaSuccess) {
      set_last_cuda_error(e);
      return DREAMS_ERR_CUDA;
    }
  }
  if (lists * nsplit > INT_MAX) return DREAMS_ERR_UNSUPPORTED;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(lists * nsplit));
  cfg.blockDim = dim3(32 * WARPS);
  cfg.dynamicSmemBytes = size_t(smem);
  cfg.stream = stream;
  cudaLaunchAttribute attr[2] = {first};
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = unsigned(nsplit);
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = nsplit > 1 ? 2 : 1;
  void *args[] = {&p};
  const cudaError_t e = cudaLaunchKernelExC(&cfg, kernel, args);
  if (e != cudaSuccess) {
    set_last_cuda_error(e);
    return DREAMS_ERR_CUDA;
  }
  return check_launch();
}

}  // namespace win
}  // namespace dreams
