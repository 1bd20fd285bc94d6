// window.cu -- attention with a sliding window and sinks.
//
// Query t of a sequence with L committed slots is at position p = L + t (causal)
// or L + depth(t) (draft tree) and sees slot s when p - s < window or s < sinks,
// new slots only up to its own (causal) or along its ancestors (tree). The keys a
// block of query rows can see are two runs of slots, the sinks and the window of
// its first query up to its last one; the kernel numbers them 0 .. n-1 as one list,
// so sinks and window share tiles and nothing between them is read.
//
// window_rows_kernel: a CTA takes 16 query rows (token, head of the GQA group) of
// one KV head and a contiguous part of their key list; its four warps take 16-key
// tiles in turn, each with its own ring of cp.async stages, so no barrier stands
// in the stream. Scores and P V run on m16n8k16 tensor instructions with the
// running maximum and sum of each row in f32 registers. The warps' partial sums
// join in shared memory, and the parts of a split key list in distributed shared
// memory (the parts are one cluster), in a fixed order. For few rows the kernel is
// bound by reading K and V once.
#include <limits.h>
#include <math.h>

#include <algorithm>

#include "window.cuh"

namespace dreams {
namespace {

using namespace win;

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
__device__ __forceinline__ float2 ld_cluster2(uint32_t addr) {
  float2 v;
  asm volatile("ld.shared::cluster.v2.f32 {%0,%1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr) : "memory");
  return v;
}
// Does a pair of bf16 values hold an infinity or a NaN?
__device__ __forceinline__ bool nonfinite2(uint32_t x) {
  return (x & 0x7f80u) == 0x7f80u || (x & 0x7f800000u) == 0x7f800000u;
}

constexpr int RB = 16;    // query rows of a CTA
constexpr int KT = 16;    // keys of a warp's tile
constexpr int WARPS = 4;

template <int D>
struct RowsCfg {
  static constexpr int STAGES = D == 128 ? 3 : 6;
  static constexpr int ROW = D * 2;                // bytes of a key
  static constexpr int TILE = KT * ROW;            // K or V of a tile
  static constexpr int WARP_BYTES = STAGES * 2 * TILE;
  static constexpr int SMEM = WARPS * WARP_BYTES;  // at the end: WARPS partial outputs [16][D] f32 and the CTA's
  static_assert(SMEM >= (WARPS + 1) * RB * D * 4, "partials fit");
};

// What a row of the block is: its position, and for a tree its visible new slots.
struct RowInfo {
  int off;                 // position - L; -1: no row
  unsigned long long anc;  // tree: bit a = sees slot L + a
};

template <int D>
__global__ void __launch_bounds__(32 * WARPS) window_rows_kernel(const WinParams p) {
  using C = RowsCfg<D>;
  constexpr int CH = D / 8;  // 16-byte columns of a key
  extern __shared__ __align__(1024) uint8_t smem[];
  __shared__ int s_par[64];
  __shared__ RowInfo s_row[RB];
  __shared__ float2 s_ml[WARPS + 1][RB];

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  int x = blockIdx.x;
  const int split = x % p.nsplit;
  x /= p.nsplit;
  const int rb = x % p.nrb;
  x /= p.nrb;
  const int g = x % p.Hkv, b = x / p.Hkv;
  const bool reporter = rb == 0 && split == 0 && g == 0 && tid == 0;

  const int T = __ldg(p.q_len + b), L = __ldg(p.kv_len + b);
  if (T < 0 || T > p.T_max) {
    if (reporter) flag(p.status, DREAMS_DATA_BAD_TREE_LEN);
    return;
  }
  if (L < 0 || int64_t(L) + T > p.capacity) {
    if (reporter) flag(p.status, DREAMS_DATA_BAD_KV_LEN);
    return;
  }
  const int t_first = rb * RB / p.G;
  if (t_first >= T) return;  // (as do all CTAs of the cluster)
  const int t_last = ::min(T - 1, (rb * RB + RB - 1) / p.G);

  // ---- rows
  if (p.parent != nullptr) {
    int bad = 0;
    for (int i = tid; i < T; i += 32 * WARPS) {
      const int par = __ldg(p.parent + int64_t(b) * p.T_max + i);
      s_par[i] = par;
      bad |= i == 0 ? par != -1 : (par < 0 || par >= i);
    }
    if (__syncthreads_or(bad)) {
      if (reporter) flag(p.status, DREAMS_DATA_BAD_PARENT);
      return;
    }
  }
  if (tid < RB) {
    const int t = (rb * RB + tid) / p.G;
    RowInfo r{-1, 0ull};
    if (t < T) {
      r.off = t;
      if (p.parent != nullptr) r.anc = tree_row(p, s_par, L, t, r.off);
    }
    s_row[tid] = r;
  }
  __syncthreads();

  const KeyList kl = key_list(p, L, t_first, t_last);
  const int64_t per = ((int64_t(kl.n) + p.nsplit - 1) / p.nsplit + KT - 1) / KT * KT;
  const int i0 = int(::min(int64_t(kl.n), split * per)), i1 = int(::min(int64_t(kl.n), i0 + per));
  const int ntiles = (i1 - i0 + KT - 1) / KT;

  // ---- this thread's part of Q: rows lane / 4 and lane / 4 + 8
  const int r0 = lane >> 2, c0 = (lane & 3) * 2;
  uint32_t qf[D / 16][4];
  int off[2];
  unsigned long long anc[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int r = r0 + 8 * h, flat = rb * RB + r, t = flat / p.G;
    off[h] = s_row[r].off;
    anc[h] = s_row[r].anc;
    const __nv_bfloat16 *src = p.q + b * p.sb + t * p.st + int64_t(g * p.G + flat - t * p.G) * D + c0;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      qf[kk][h] = t < T ? *reinterpret_cast<const uint32_t *>(src + kk * 16) : 0u;
      qf[kk][h + 2] = t < T ? *reinterpret_cast<const uint32_t *>(src + kk * 16 + 8) : 0u;
    }
  }

  // ---- the stream of this warp: tiles warp, warp + WARPS, ...
  const uint32_t ring = smem_u32(smem) + warp * C::WARP_BYTES;
  const int my = ntiles > warp ? (ntiles - warp + WARPS - 1) / WARPS : 0;
  // lane k (mod 16) looks after key k of a tile: its slot and page entry one
  // tile ahead of the copy
  int nslot = -1, npage = 0;
  auto look = [&](int j) {
    const int i = i0 + (warp + j * WARPS) * KT + (lane & 15);
    nslot = j < my && i < i1 ? kl.slot(i) : -1;
    if (p.table != nullptr && nslot >= 0) npage = __ldg(p.table + int64_t(b) * p.P + (nslot >> 6));
  };
  auto issue = [&](int j) {
    if (j < my) {
      int64_t at = -1;
      if (nslot >= 0) {
        if (p.table == nullptr) {
          at = (int64_t(b) * p.capacity + nslot) * p.Hkv + g;
        } else if (npage >= 0 && npage < p.num_pages) {
          at = (int64_t(npage) * 64 + (nslot & 63)) * p.Hkv + g;
        } else if (lane < 16) {
          flag(p.status, DREAMS_DATA_BAD_PAGE);
        }
      }
      look(j + 1);
      const uint32_t st = ring + (j % C::STAGES) * 2 * C::TILE;
#pragma unroll
      for (int it = 0; it < KT * CH / 32; ++it) {
        const int u = it * 32 + lane, key = u / CH, ch = u % CH;
        const int64_t o = __shfl_sync(0xffffffffu, at, key);
        const uint32_t dst = st + key * C::ROW + ((ch ^ (key & 7)) << 4);
        const int64_t e = o < 0 ? 0 : o * D + ch * 8;
        const int bytes = o < 0 ? 0 : 16;
        cp_async16(dst, p.k + e, bytes);
        cp_async16(dst + C::TILE, p.v + e, bytes);
      }
    }
    cp_commit();
  };
  look(0);
#pragma unroll
  for (int j = 0; j < C::STAGES - 1; ++j) issue(j);

  float o[D / 8][4];
#pragma unroll
  for (int n = 0; n < D / 8; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};

  const int off_min = p.parent != nullptr ? 0 : t_first, off_max = t_last;
  for (int j = 0; j < my; ++j) {
    cp_wait<C::STAGES - 2>();
    __syncwarp();
    issue(j + C::STAGES - 1);
    const uint32_t st = ring + (j % C::STAGES) * 2 * C::TILE;
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
                       (p.parent != nullptr ? sl < L : sl <= L + off_min)));
    if (!all) {
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = ib + n * 8 + c0 + (e & 1);
          if (i >= i1 || off[e >> 1] < 0 || !sees(p, L, off[e >> 1], anc[e >> 1], kl.slot(i))) s[n][e] = -INFINITY;
        }
    }
    uint32_t pf[4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float mx = fmaxf(fmaxf(s[0][2 * h], s[0][2 * h + 1]), fmaxf(s[1][2 * h], s[1][2 * h + 1]));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
      mx *= p.scale_log2;
      const float mn = fmaxf(m[h], mx);
      if (mn > m[h]) {  // the same in the four threads of a row
        const float corr = tc::ex2(m[h] - mn);
        l[h] *= corr;
#pragma unroll
        for (int n = 0; n < D / 8; ++n) {
          o[n][2 * h] *= corr;
          o[n][2 * h + 1] *= corr;
        }
        m[h] = mn;
      }
      const float nm = mn == -INFINITY ? 0.f : -mn;
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const float p0 = tc::ex2(fmaf(s[n][2 * h], p.scale_log2, nm));
        const float p1 = tc::ex2(fmaf(s[n][2 * h + 1], p.scale_log2, nm));
        l[h] += p0 + p1;
        pf[2 * n + h] = pack_bf16x2(p0, p1);
      }
    }
    // O += P V
    {
      const int key = (((lane >> 3) & 1) << 3) + (lane & 7), half = lane >> 4;
#pragma unroll
      for (int n = 0; n < D / 8; n += 2) {
        uint32_t vb[4];
        ldsm4t(st + C::TILE + key * C::ROW + (((n + half) ^ (key & 7)) << 4), vb);
        // 0 x inf and 0 x NaN are NaN: where a key that not every row sees holds
        // one, each row takes its product from its own keys alone
        if (!all && __any_sync(0xffffffffu, nonfinite2(vb[0]) || nonfinite2(vb[1]) || nonfinite2(vb[2]) || nonfinite2(vb[3]))) {
#pragma unroll 1
          for (int r = 0; r < RB; ++r) {
            const RowInfo ri = s_row[r];
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
            float a0[4] = {0.f, 0.f, 0.f, 0.f}, a1[4] = {0.f, 0.f, 0.f, 0.f};
            mma16816(a0, pf, vb[0] & keep[0], vb[1] & keep[1]);
            mma16816(a1, pf, vb[2] & keep[0], vb[3] & keep[1]);
#pragma unroll
            for (int h = 0; h < 2; ++h)
              if (r0 + 8 * h == r) {
                o[n][2 * h] += a0[2 * h];
                o[n][2 * h + 1] += a0[2 * h + 1];
                o[n + 1][2 * h] += a1[2 * h];
                o[n + 1][2 * h + 1] += a1[2 * h + 1];
              }
          }
        } else {
          mma16816(o[n], pf, vb[0], vb[1]);
          mma16816(o[n + 1], pf, vb[2], vb[3]);
        }
      }
    }
  }
  cp_wait<0>();
  __syncthreads();  // the stages are free

  // ---- the warps' parts, then the CTA's: [warp][row][D] and (m, l)
  float *so = reinterpret_cast<float *>(smem);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
    l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
    const int r = r0 + 8 * h;
    if ((lane & 3) == 0) s_ml[warp][r] = make_float2(m[h], l[h]);
#pragma unroll
    for (int n = 0; n < D / 8; ++n)
      *reinterpret_cast<float2 *>(so + (warp * RB + r) * D + n * 8 + c0) = make_float2(o[n][2 * h], o[n][2 * h + 1]);
  }
  __syncthreads();
  const bool whole = p.nsplit == 1;
  auto emit = [&](int r, int d, float2 v, float M, float Z) {
    const int flat = rb * RB + r, t = flat / p.G;
    if (t >= T) return;
    const int64_t row = (int64_t(b) * p.T_max + t) * p.Hq + g * p.G + (flat - t * p.G);
    const float inv = 1.f / Z;
    *reinterpret_cast<uint32_t *>(p.out + row * D + d) = pack_bf16x2(v.x * inv, v.y * inv);
    if (d == 0 && p.lse != nullptr) p.lse[row] = (M + log2f(Z)) * LN2;
  };
  float *sc = so + WARPS * RB * D;  // the CTA's part
#pragma unroll 1
  for (int u = tid; u < RB * D / 2; u += 32 * WARPS) {
    const int r = u / (D / 2), d = (u - r * (D / 2)) * 2;
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) M = fmaxf(M, s_ml[w][r].x);
    float Z = 0.f;
    float2 acc = make_float2(0.f, 0.f);
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
      const float2 ml = s_ml[w][r];
      if (ml.y == 0.f) continue;  // no key (a NaN sum goes through)
      const float c = tc::ex2(ml.x - M);
      const float2 ov = *reinterpret_cast<const float2 *>(so + (w * RB + r) * D + d);
      Z += c * ml.y;
      acc.x += c * ov.x;
      acc.y += c * ov.y;
    }
    if (whole) {
      emit(r, d, acc, M, Z);
    } else {
      *reinterpret_cast<float2 *>(sc + r * D + d) = acc;
      if (d == 0) s_ml[WARPS][r] = make_float2(M, Z);
    }
  }
  if (whole) return;

  // ---- the parts of a split list: each CTA of the cluster joins its share of
  // the outputs from all of them
  cluster_sync();
  const uint32_t ml_a = smem_u32(&s_ml[WARPS][0]), sc_a = smem_u32(sc);
  for (int u = split * 32 * WARPS + tid; u < RB * D / 2; u += p.nsplit * 32 * WARPS) {
    const int r = u / (D / 2), d = (u - r * (D / 2)) * 2;
    float M = -INFINITY;
    for (int c = 0; c < p.nsplit; ++c) M = fmaxf(M, ld_cluster2(mapa(ml_a + r * 8, c)).x);
    float Z = 0.f;
    float2 acc = make_float2(0.f, 0.f);
    for (int c = 0; c < p.nsplit; ++c) {
      const float2 ml = ld_cluster2(mapa(ml_a + r * 8, c));
      if (ml.y == 0.f) continue;
      const float w = tc::ex2(ml.x - M);
      const float2 ov = ld_cluster2(mapa(sc_a + (r * D + d) * 4, c));
      Z += w * ml.y;
      acc.x += w * ov.x;
      acc.y += w * ov.y;
    }
    emit(r, d, acc, M, Z);
  }
  cluster_sync();  // no CTA leaves while another reads its shared memory
}

// ------------------------------------------------------------------ host side
template <int D>
dreams_status_t launch_rows(WinParams p, cudaStream_t stream) {
  const void *kernel = reinterpret_cast<const void *>(window_rows_kernel<D>);
  const dreams_status_t st = ensure_max_dynamic_smem(kernel, RowsCfg<D>::SMEM);
  if (st != DREAMS_OK) return st;
  p.nrb = int((int64_t(p.T_max) * p.G + RB - 1) / RB);
  const int64_t items = int64_t(p.B) * p.Hkv * p.nrb;
  // keys a block can see at most
  const int64_t keys = std::min<int64_t>(p.capacity, int64_t(p.window) + p.sinks + std::min<int64_t>(p.T_max, RB));
  p.nsplit = 1;
  while (p.nsplit < 8 && items * p.nsplit < 4 * int64_t(num_sms()) && keys / p.nsplit > 2 * WARPS * KT) p.nsplit *= 2;
  if (items * p.nsplit > INT_MAX) return DREAMS_ERR_UNSUPPORTED;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(items * p.nsplit));
  cfg.blockDim = dim3(32 * WARPS);
  cfg.dynamicSmemBytes = RowsCfg<D>::SMEM;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = unsigned(p.nsplit);
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = p.nsplit > 1 ? 1 : 0;
  void *args[] = {&p};
  const cudaError_t e = cudaLaunchKernelExC(&cfg, kernel, args);
  if (e != cudaSuccess) {
    set_last_cuda_error(e);
    return DREAMS_ERR_CUDA;
  }
  return check_launch();
}

bool shapes_ok(const dreams_kv_cache_t *kv, int32_t B, int32_t T_max, int32_t Hq, int32_t window, int32_t sinks,
               bool tree) {
  return kv != nullptr && B >= 1 && B <= 65535 && T_max >= 1 && T_max <= (tree ? 64 : 1 << 20) && kv->Hkv >= 1 &&
         kv->Hkv <= 65535 && Hq >= kv->Hkv && Hq % kv->Hkv == 0 && Hq / kv->Hkv <= 128 && kv->capacity >= 1 &&
         kv->n_layers >= 1 && window >= 1 && sinks >= 0;
}

}  // namespace
}  // namespace dreams

using namespace dreams;

extern "C" size_t dreams_window_attention_workspace_size(const dreams_kv_cache_t *kv, int32_t B, int32_t T_max,
                                                         int32_t Hq, int32_t window, int32_t sinks, int32_t tree) {
  if (!shapes_ok(kv, B, T_max, Hq, window, sinks, tree != 0)) return 0;
  return 0;
}

extern "C" dreams_status_t dreams_window_attention(const void *q, int64_t q_stride_b, int64_t q_stride_t,
                                                   const dreams_kv_cache_t *kv, int32_t layer, const int32_t *parent,
                                                   const int32_t *q_len, const int32_t *kv_len, int32_t B,
                                                   int32_t T_max, int32_t Hq, float scale, int32_t window,
                                                   int32_t sinks, void *out, float *lse, void *workspace,
                                                   size_t workspace_bytes, int32_t *status_word,
                                                   dreams_stream_t stream) {
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
  if (B == 1) q_stride_b = q_stride_t;  // not used
  if (q_stride_t < int64_t(Hq) * kv->D || q_stride_b < int64_t(Hq) * kv->D || q_stride_t % 8 != 0 ||
      q_stride_b % 8 != 0 || q_stride_t >= (int64_t(1) << 38) || q_stride_b >= (int64_t(1) << 38))
    return DREAMS_ERR_INVALID_ARG;
  if (kv->page_table != nullptr) {
    if (kv->page_size != 64) return DREAMS_ERR_UNSUPPORTED;
    if (kv->pages_per_seq < 1 || kv->num_pages < 1 || int64_t(kv->pages_per_seq) * 64 != kv->capacity)
      return DREAMS_ERR_INVALID_ARG;
  }
  WinParams p{};
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
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (int64_t(T_max) * p.G > RB) return launch_tc(p, kv, s);
  return kv->D == 128 ? launch_rows<128>(p, s) : launch_rows<64>(p, s);
}
