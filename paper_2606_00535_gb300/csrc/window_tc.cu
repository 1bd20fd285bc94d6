// window_tc.cu -- windowed attention for blocks of 128 query rows on tcgen05
// tensor cores (prefill, chunks, draft trees).
//
// A block is 128 / G tokens times the G query heads of a KV head. Its keys are a row of
// 64-slot pages: those of the sinks first, then the window of the block's first query
// up to its last one. Two pages make a tile; the last one is cut to the columns it
// needs (a multiple of 32). A few sinks so cost half a tile (as a tile of their own
// they cost more than a full one: 2500 tokens with window 700 55 us, now 48).
//
// One CTA per SM holds two slots of tensor memory (256 columns: S, then P, and O).
// S = Q K^T and O += P V are tcgen05 groups; a slot's softmax warpgroup, one row per
// thread, turns S into P and hands it over in two halves, so that the first half of
// P V runs under the second. The slots' chains interleave on the tensor pipe. With
// head dim 64 P lies beside S, and the next Q K^T starts when S has been read.
//
// Softmax without a running maximum: a row's reference m is the maximum of the first
// tile it sees a key of, and stays; P = 2^(x - m) is as exact at any m, in bf16 and in
// the f32 sums alike, short of overflow. So the exponentials of a tile start as its
// scores arrive. P enters P V as one bf16: the outputs' error against 64 bits is then 1.2
// to 1.4 times that of f32 probabilities (the one rounding of the output is most of
// either), and a product with what is left of P would add half of Q K^T and P V to the
// tensor pipe. A row whose sum ends above 2^100 (a later score exceeds m by some 69
// nats), or above 2^40 (28 nats) with an O that overflowed, is done again from its
// definition.
//   PAIR   the slots are two neighbouring blocks of a KV head: every K/V tile is
//          loaded once for 256 rows. The CTAs are persistent: they walk over the
//          items with a ring of K/V stages that runs on across them, so the next
//          item's loads and first Q K^T overlap the epilogue of the last.
//   CLUSTER  pairs over 8-bit pages, on clusters of two CTAs: pair A, one of the longest, is cut
//          so that the first CTA's part of it is as long as the second's and pair B, one
//          of the shortest, together; A's parts are joined through distributed shared memory.
//   !PAIR  both slots work on one block, alternate tiles; a block's tiles may be
//          split over a cluster of CTAs, joined through distributed shared memory.
//          For grids too small to fill the SMs with pairs.
// Warps: 0-3 and 4-7 the softmax of slots 0 and 1, 8 the TMA producer, 9 and 10 the
// MMA issuers of the slots (one thread each, so that one's waits run under the
// other's MMAs), 11 the scan (below), which also zeroes the V rows that nobody sees. A
// slot's MMAs complete in order, so the commit that announces S of a tile also says
// that the P V before it is done: the softmax warpgroup then gives those stages back,
// and no further commits are needed.
//   EIGHT  pages below a sequence's len8 come as codes, and four warps more, 12-15, turn
//          them into bf16 between the copy and everything else (a code times its page's
//          power of two is exact in bf16). They take about 1200 clocks of a tile of 4400 and
//          slow the softmax, whose schedulers they share, from 2000 to 2500 (head dim 64: 2500
//          to 3200): the bytes are half, and the time 10 to 15% above that of the
//          same pairs in bf16. Work is laid out anew instead: pairs in order of their tiles,
//          or cut between two CTAs (CLUSTER). 16 trees of up to 64 nodes on 1500 to 6000 tokens,
//          32/8 heads: 93 us (as in bf16, one pair a CTA: 112); four chunks of 701 to 999
//          tokens on as many, head dim 64: 213 us (pairs as they come: 255).
// Bound by the chain of a tile (products, softmax, products), of which two run on an
// SM: about 4000 clocks for both slots, where the products take 2048, with head dim 128
// (1.93 us a tile of a pair at 2070 MHz, from windows of 2048 to 8192); 2900 with head
// dim 64 (1.41 us), where products and exponentials take 1024 each. 3392 tokens of 32
// heads, head dim 128, window 1024: 73 us, 35% of the bf16 burst rate on the keys seen;
// 16 trees of up to 64 nodes, 32/8 heads, window 2048: 45 us, 48% of the copy rate.
// Every mbarrier wait is bounded (2 s without progress); a CTA that gives up flags DREAMS_DATA_TIMEOUT,
// drains its copies and MMAs, frees its tensor memory and leaves unfinished rows
// untouched.
#include <cuda.h>
#include <limits.h>
#include <math.h>
#include <string.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "tmap.cuh"
#include "kv8.cuh"
#include "window.cuh"

namespace dreams {
namespace win {
namespace {

constexpr int KT = 128;    // keys of a tile
constexpr int ROWS = 128;  // query rows of a block
constexpr int TMA_WARP = 8, MMA_WARP = 9, SCAN_WARP = 11;  // slot w's MMAs: warp MMA_WARP + w
constexpr int CODE_WARP = 12, CODE_WARPS = 4;              // EIGHT: those that turn codes into bf16
// Items whose scan results are kept: more than the scan can be ahead of a slot that has
// tiles of the item, as it needs stages which that slot gives back. Of a slot that has
// none it can be ahead by any number of items, so such a slot asks for no result.
constexpr int SEEN = 16;
constexpr uint32_t TMEM_COLS = 512;
// A row whose sum ends above MOST_SUM (2^100) is done again, and so is one whose O has
// overflowed with a sum above SAFE_SUM (2^40). |O| is at most the sum times the largest
// |V|, so below that sum no O overflows for |V| up to 2^87, and above it an infinity or
// a NaN of O may not be V's.
constexpr float MOST_SUM = 1.2676506e30f, SAFE_SUM = 1.0995116e12f;

template <int D, bool PAIR, bool EIGHT>
struct Cfg {
  static constexpr int THREADS = EIGHT ? 512 : 384;
  static constexpr int NR = D / 64;  // 128-byte column regions of a row
  static constexpr uint32_t Q_REGION = ROWS * 128, KV_REGION = KT * 128;
  static constexpr uint32_t Q_BYTES = NR * Q_REGION;
  static constexpr uint32_t STAGE = NR * KV_REGION;
  static constexpr int NQ = PAIR ? 2 : 1;
  // A slot's columns: S at 0; with head dim 64 there is room for P beside it, and the
  // next Q K^T can start once the scores are in registers; with 128 P goes over S.
  static constexpr bool BESIDE = D == 64;
  static constexpr uint32_t P_COL = BESIDE ? 128 : 0, O_COL = BESIDE ? 192 : 128;
  // (Six stages for single blocks over 8-bit pages, whose two slots hold four: 512 blocks on
  // 1500 to 6000 tokens 279 us, 305 with five; one tree on 7808 47.2, 49.2.)
  static constexpr int NST = D == 64 ? 8 : EIGHT && !PAIR ? 6 : 5;
  // EIGHT: where a stage's codes land, two pages HALF bytes apart. With head dim 128 a row's
  // lie in the stage itself, where its first 64 dimensions come to lie, so that a warp
  // writes over its own rows' alone; with 64 there is room beside it.
  static constexpr bool IN_PLACE = D == 128;
  static constexpr uint32_t HALF = IN_PLACE ? 8192 : 64 * D, CODES = IN_PLACE ? STAGE : 2 * HALF;
  static constexpr size_t SMEM = std::max<size_t>(NQ * Q_BYTES + size_t(NST) * (STAGE + (EIGHT && !IN_PLACE ? CODES : 0)) + 1024, 120 * 1024);
};

struct TcParams {
  CUtensorMap tmap_q, tmap_k, tmap_v;
  WinParams p;
  int32_t TB;      // tokens of a block
  int32_t nblk;    // blocks (or pairs) per sequence and KV head
  int32_t items;   // B * Hkv * nblk
  Divisor heads, hkv, nsplit, g;  // B * Hkv, Hkv, CTAs of a cluster, query heads per KV head
  int32_t stall_at;
  uint64_t wait_ns;
};
struct Tc8Params : TcParams {
  CUtensorMap tmap_k8, tmap_v8;
  Kv8 c;
  Divisor seqs;    // B
  int32_t ranked;    // pairs: those with the most tiles first
  int32_t clusters;  // CLUSTER: that run at once
};
template <bool EIGHT>
using ParamsOf = std::conditional_t<EIGHT, Tc8Params, TcParams>;

// An item: a pair of blocks, or one block, of a sequence and KV head. Its keys are
// np half tiles of up to 64 slots, the nsp sink ones first; tile j is the halves
// 2j and 2j + 1. A key's column is its place in that row of halves.
struct Item {
  int b, g, L, T, L8;      // L8: slots in 8 bits
  int t00, t01, tl0, tl1;  // first and last token of each block
  int nb;                  // blocks present (0: nothing to do)
  int lo, lo64, S1, hi;
  int nsp, np, ns, n;      // ns: tiles with sinks
  int e0, a1;              // block 0 reads tiles [0, e0), block 1 [0, ns) and [a1, n)
  __device__ __forceinline__ bool need0(int j) const { return j < e0; }
  __device__ __forceinline__ bool need1(int j) const { return nb == 2 && j < n && (j < ns || j >= a1); }
  __device__ __forceinline__ bool codes(int q) const { return q < np && slot0(q) < L8; }
  __device__ __forceinline__ int slot0(int q) const { return q < nsp ? q * 64 : lo64 + (q - nsp) * 64; }
  // the slots of half q that a row may see, from its first one on
  __device__ __forceinline__ int beg(int q) const { return q < nsp ? 0 : ::max(0, lo - slot0(q)); }
  __device__ __forceinline__ int end(int q) const { return ::min(64, (q < nsp ? S1 : hi) - slot0(q)); }
  __device__ __forceinline__ bool part(int q) const { return beg(q) > 0 || end(q) < 64; }
  __device__ __forceinline__ bool cut(int j) const { return part(2 * j) || (2 * j + 1 < np && part(2 * j + 1)); }
  __device__ __forceinline__ int column(int slot) const { return nsp * 64 + slot - lo64; }  // of the window's run
  __device__ __forceinline__ int ncols(int j) const { return ::min(KT, (column(hi) - j * KT + 31) & ~31); }
};

// The first tile of each split; some are one longer, the first one last (it has the tile
// with the sinks), but the first splits are those with tiles.
struct Splits {
  int each, longer;
  __device__ __forceinline__ Splits(int n, const Divisor &of) : each(of.div(n)), longer(n - each * int(of.d)) {}
  __device__ __forceinline__ int first(int split) const { return split * each + ::min(each > 0 ? ::max(split - 1, 0) : split, longer); }
};

// The tiles that every row of a block sees whole: [0, sink) and [from, to).
struct Whole {
  int sink, from, to;
  __device__ __forceinline__ bool operator()(int j) const { return j < sink || (j >= from && j < to); }
};
__device__ __forceinline__ Whole whole_tiles(const WinParams &p, const Item &it, int w) {
  const int t0 = w ? it.t01 : it.t00, tl = w ? it.tl1 : it.tl0;
  const int from = ::max(it.lo, it.L + tl - p.window + 1) - it.lo64;                              // >= 0
  const int to = ::min(it.hi, p.parent != nullptr ? it.L : it.L + t0 + 1) - it.lo64;
  return Whole{it.S1 / KT, (it.nsp + (from + 63) / 64 + 1) / 2, (it.nsp + (to > 0 ? to / 64 : 0)) / 2};
}

// What is known of a sequence.
struct Lens {
  int T, L, L8;
};
template <bool EIGHT>
__device__ __forceinline__ Lens lens_of(const ParamsOf<EIGHT> &P, int b) {
  Lens l{P.p.q_len[b], P.p.kv_len[b], 0};
  if constexpr (EIGHT) l.L8 = P.c.len8[b];
  return l;
}

template <bool PAIR, bool EIGHT>
__device__ __forceinline__ void load_item(const ParamsOf<EIGHT> &P, int blk, Item &it, bool report, const Lens *lens) {
  const WinParams &p = P.p;
  const Lens l = lens != nullptr ? *lens : lens_of<EIGHT>(P, it.b);
  it.T = l.T;
  it.L = l.L;
  it.L8 = l.L8;
  it.nb = it.n = it.ns = 0;
  report = report && it.g == 0 && blk == 0;
  if (it.T < 0 || it.T > p.T_max) {
    if (report) flag(p.status, DREAMS_DATA_BAD_TREE_LEN);
    return;
  }
  bool odd = it.L < 0 || int64_t(it.L) + it.T > p.capacity;
  if constexpr (EIGHT) odd = odd || len8_bad(P.c, it.L8, it.L);
  if (odd) {
    if (report) flag(p.status, DREAMS_DATA_BAD_KV_LEN);
    return;
  }
  it.t00 = blk * (PAIR ? 2 : 1) * P.TB;
  it.t01 = it.t00 + P.TB;
  if (it.t00 >= it.T) return;
  it.nb = PAIR && it.t01 < it.T ? 2 : 1;
  it.tl0 = ::min(it.T, it.t00 + P.TB) - 1;
  it.tl1 = it.nb == 2 ? ::min(it.T, it.t01 + P.TB) - 1 : it.tl0;
  const bool tree = p.parent != nullptr;
  it.lo = ::max(0, it.L + (tree ? 0 : it.t00) - p.window + 1);
  // with more sinks than slots before the window, all slots are one run
  const bool one_run = p.sinks > it.lo;
  if (one_run) it.lo = 0;
  it.S1 = one_run ? 0 : p.sinks;
  it.lo64 = it.lo & ~63;
  it.nsp = (it.S1 + 63) / 64;
  it.ns = (it.nsp + 1) / 2;
  it.hi = it.L + it.tl1 + 1;
  it.np = it.nsp + (it.hi - it.lo64 + 63) / 64;
  it.n = (it.np + 1) / 2;
  const int lo1 = ::max(0, it.L + (tree ? 0 : it.t01) - p.window + 1);
  it.a1 = one_run ? 0 : ::max(it.ns, (it.nsp + (lo1 - it.lo64) / 64) / 2);
  it.e0 = (it.nsp + (it.L + it.tl0 - it.lo64) / 64) / 2 + 1;
}

// EIGHT: the pairs of blocks of all sequences in order of their tiles, most first.
constexpr int MAX_RANKED = 256;
// CLUSTER: what a change of items costs, and the least part that is worth a join, in tiles.
// (The least 8: 12 trees on 300 to 1500 tokens 39.6 us, 30.8 with 4; 2: 16 on 2000 to 3000
// 72.1, 69.9 with 4. A change 5: 16 on 1500 to 6000 98.6, 93.8 with 2; 0: 92.7, but head dim
// 64 on 300 to 1500 35.4 for 33.9.)
constexpr int CHANGE = 2, LEAST = 4;
__device__ __forceinline__ void rank_items(const Tc8Params &P, int *tiles, uint8_t *order) {  // tiles: of entry i, for what follows too
  const int i = threadIdx.x, n = P.nblk * P.p.B;
  int mine = -1;
  if (i < n) {
    Item it;
    const int turn = P.seqs.div(i);
    it.b = i - turn * P.p.B;
    it.g = 0;
    load_item<true, true>(P, P.nblk - 1 - turn, it, false, nullptr);
    mine = it.nb > 0 ? it.n : 0;
  }
  if (i < MAX_RANKED) tiles[i] = mine;
  tc::fence_proxy_async_smem();  // (copies will land there)
  __syncthreads();
  if (i < n) {
    int before = 0;
#pragma unroll 4
    for (int k = 0; 4 * k < n; ++k) {
      const int4 x = reinterpret_cast<const int4 *>(tiles)[k];
      before += int(x.x > mine || (x.x == mine && 4 * k < i)) + int(x.y > mine || (x.y == mine && 4 * k + 1 < i)) +
                int(x.z > mine || (x.z == mine && 4 * k + 2 < i)) + int(x.w > mine || (x.w == mine && 4 * k + 3 < i));
    }
    order[before] = uint8_t(i);
  }
}

// An arrival by the threads for which `yes` holds, without a branch.
__device__ __forceinline__ void arrive_if(uint32_t bar, bool yes) {
  asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %1, 0;\n @p mbarrier.arrive.shared::cta.b64 _, [%0];\n}\n" ::"r"(bar), "r"(int(yes)) : "memory");
}

// What the rows of an item see: columns [0, sinks) and from their window's first one
// on, in a tree up to those of the new slots, of which a row sees its ancestors.
struct View {
  int first, lowest;  // first column of the window at offset 0; no row's is lower
  int fresh, sinks;   // column of slot L; sinks
};

// What a softmax warp keeps of an item in shared memory.
struct __align__(16) Slot {
  View view;
  int L, cols, t0, rows, b, g, bad;
};

// A place in the ring of stages: index and phase.
template <int N>
struct Place {
  int s;
  uint32_t ph;
  __device__ __forceinline__ Place plus(int d) const {  // d < N
    Place q{s + d, ph};
    if (q.s >= N) {
      q.s -= N;
      q.ph ^= 1u;
    }
    return q;
  }
  __device__ __forceinline__ void move(int d) {  // any d >= 0
    const uint32_t at = uint32_t(s + d), q = at / N;
    s = int(at - q * N);
    ph ^= q & 1u;
  }
};

__device__ __forceinline__ uint64_t f32x2(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void f32x2_split(uint64_t v, float &lo, float &hi) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ uint64_t ffma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t fadd2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ float4 ld_cluster4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ float2 ld_cluster2(uint32_t addr) {
  float2 v;
  asm volatile("ld.shared::cluster.v2.f32 {%0,%1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void st_cluster(uint32_t addr, uint32_t v) { asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory"); }
__device__ __forceinline__ void st_cluster2(uint32_t addr, float2 v) {
  asm volatile("st.shared::cluster.v2.f32 [%0], {%1,%2};" ::"r"(addr), "f"(v.x), "f"(v.y) : "memory");
}
__device__ __forceinline__ void st_cluster4(uint32_t addr, const uint32_t *v) {
  asm volatile("st.shared::cluster.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
}
// tcgen05.mma of kind::f16 with the descriptors' low words in registers: the high
// word (stride offset 1024 bytes, 128-byte swizzle) is the same for every operand.
constexpr uint32_t DESC_HI = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n .reg .pred p;\n .reg .b64 a, b;\n setp.ne.b32 p, %4, 0;\n mov.b64 a, {%1, %5};\n mov.b64 b, {%2, %5};\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n}\n" ::"r"(d),
      "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(acc), "n"(DESC_HI)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b_lo, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n .reg .pred p;\n .reg .b64 b;\n setp.ne.b32 p, %4, 0;\n mov.b64 b, {%2, %5};\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n}\n" ::"r"(d),
      "r"(a), "r"(b_lo), "r"(idesc), "r"(acc), "n"(DESC_HI)
      : "memory");
}
// tc::mbar_wait with a hint that lets the hardware suspend the warp for longer: a
// spinning warp takes issue slots from the softmax warps of its scheduler.
__device__ __forceinline__ bool try_wait(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n selp.u32 %0, 1, 0, p;\n}\n"
               : "=r"(ok)
               : "r"(bar), "r"(parity), "r"(20000u)
               : "memory");
  return ok != 0;
}
// Waiting for what has happened takes half as long without the hint (135 clocks
// against 270), and an MMA issuer does it four times a tile.
__device__ __forceinline__ bool quick(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}\n" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
// The limit is one without progress: rows that a warp does again key by key may take
// longer than that, and the CTA's other warps wait for them. `beat` is the last time that
// such a warp gave. The loop is out of line, as few waits outlast the first two tries.
__device__ __noinline__ bool patient(uint32_t bar, uint32_t parity, volatile int *abort, volatile int64_t *beat, uint64_t limit_ns) {
  uint64_t t0 = 0;
  for (;;) {
    if (try_wait(bar, parity)) return true;
    const uint64_t now = tc::global_ns();
    if (t0 == 0) t0 = now;
    if (*abort || (now - t0 > limit_ns && int64_t(now) - *beat > int64_t(limit_ns))) return false;
  }
}
__device__ __forceinline__ bool long_wait(uint32_t bar, uint32_t parity, volatile int *abort, volatile int64_t *beat, uint64_t limit_ns) {
  return quick(bar, parity) || try_wait(bar, parity) || patient(bar, parity, abort, beat, limit_ns);
}
__device__ __forceinline__ void st_global_v8(void *p, const uint32_t *v) {
  asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}
// The low n bits of a word (n may be any integer).
__device__ __forceinline__ uint32_t low_bits(int n) {
  uint32_t r;
  asm("shl.b32 %0, %1, %2;" : "=r"(r) : "r"(0xffffffffu), "r"(::max(n, 0)));  // (a shift by 32 or more leaves nothing)
  return ~r;
}

// A lane's codes of 16 rows of a page (16 of each of 16 / RS) times 2^e, as bf16 into
// the ring: `from` its first 8 codes, the other 8 `flip` bytes on; `to` where they go.
// A warp has all of its rows' codes in registers before it writes over them.
__device__ __forceinline__ uint32_t factor_of(int e) {  // 2^(120 + e), e <= 7, or NaN; twice
  const uint32_t f = e == DREAMS_KV8_NOT_FINITE ? 0x7fffu : uint32_t(247 + ::max(e, -247)) << 7;
  return f | f << 16;
}
template <int D, int N>
__device__ __forceinline__ void fetch_codes(uint32_t from, uint32_t flip, uint32_t (&u)[N][4]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    asm volatile("ld.shared.v2.b32 {%0,%1}, [%2];" : "=r"(u[i][0]), "=r"(u[i][1]) : "r"(from + 512 * i) : "memory");
    asm volatile("ld.shared.v2.b32 {%0,%1}, [%2];" : "=r"(u[i][2]), "=r"(u[i][3]) : "r"(from + 512 * i + flip) : "memory");
  }
}
template <int D, uint32_t HALF>
__device__ __forceinline__ void widen(uint32_t from, uint32_t to, int e0, int e1, uint32_t flip) {  // of two pages
  constexpr int RS = 32 / (D / 16), N = 16 / RS;  // rows side by side (512 bytes); rows of a lane
  uint32_t u[2][N][4];
  fetch_codes<D>(from, flip, u[0]);
  fetch_codes<D>(from + HALF, flip, u[1]);
  __syncwarp();
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t up = factor_of(h == 0 ? e0 : e1);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      uint32_t v[8];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        v[2 * k] = mul_bf16x2(codes_x2<sel_of(0, 1)>(u[h][i][k]), up);
        v[2 * k + 1] = mul_bf16x2(codes_x2<sel_of(2, 3)>(u[h][i][k]), up);
      }
      // (rows 4 on have the third bit of their swizzle turned)
      const uint32_t dst = (to ^ (RS == 4 && (i & 1) ? 64u : 0u)) + 8192 * h + RS * 128 * i;
      asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(dst), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
      asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(dst ^ 16u), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
    }
  }
}
// The same for one page, of any power: beyond 2^7 the factor is beyond bf16, and comes in two.
template <int D>
__device__ __noinline__ void widen_rare(uint32_t from, uint32_t to, int e, uint32_t flip) {
  constexpr int RS = 32 / (D / 16), N = 16 / RS;
  const bool large = e > 7 && e != DREAMS_KV8_NOT_FINITE;
  const uint32_t up = large ? 0x7f007f00u : factor_of(e), f2 = large ? uint32_t(::min(120 + e, 254)) << 7 : 0x3f80u, up2 = f2 | f2 << 16;
  uint32_t u[N][4];
  fetch_codes<D>(from, flip, u);
  __syncwarp();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint32_t dst = (to ^ (RS == 4 && (i & 1) ? 64u : 0u)) + RS * 128 * i;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const uint32_t a = u[i][2 * k], b = u[i][2 * k + 1];
      asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(dst ^ (16u * k)), "r"(mul_bf16x2(mul_bf16x2(codes_x2<sel_of(0, 1)>(a), up), up2)),
                   "r"(mul_bf16x2(mul_bf16x2(codes_x2<sel_of(2, 3)>(a), up), up2)), "r"(mul_bf16x2(mul_bf16x2(codes_x2<sel_of(0, 1)>(b), up), up2)),
                   "r"(mul_bf16x2(mul_bf16x2(codes_x2<sel_of(2, 3)>(b), up), up2))
                   : "memory");
    }
  }
}

// A query row: its position (less L) and, in a tree, the new slots it sees.
struct Row {
  int off;
  unsigned long long anc;
};

// One row by a whole warp, straight from the definition: used when a tile with
// partly masked columns held an infinity or a NaN in V (0 x inf would reach rows
// that do not see it), and when a row's sum outgrew its reference. Slow (0.58 us a key,
// a chain of page entry, K, five shuffles and exponentials), and rare; `beat` is given the
// time while it lasts.
template <int D, bool EIGHT>
__device__ __noinline__ void slow_row(const ParamsOf<EIGHT> &P, int b, int g, int L, int t, int h, int off, unsigned long long anc,
                                      volatile int64_t *beat) {
  const WinParams &p = P.p;
  const int lane = threadIdx.x & 31;
  constexpr int E = D / 32;
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
    if ((i & 63) == 0 && lane == 0) *beat = int64_t(tc::global_ns());
    const int s = kl.slot(i);
    if (!sees(p, L, off, anc, s)) continue;
    int64_t at;
    bool codes = false;
    uint32_t exps = 0;
    if constexpr (EIGHT) codes = s < P.c.len8[b];
    if (codes) {
      if constexpr (EIGHT) {
        const int pg = P.c.table[int64_t(b) * P.c.P + (s >> 6)];
        at = pg >= 0 && pg < P.c.num_pages ? (int64_t(pg) * 64 + (s & 63)) * p.Hkv + g : -1;
        if (at >= 0) exps = P.c.exps[int64_t(pg) * p.Hkv + g];
      }
    } else if (p.table == nullptr) {
      at = (int64_t(b) * p.capacity + s) * p.Hkv + g;
    } else {
      const int pg = p.table[int64_t(b) * p.P + (s >> 6)];
      at = pg >= 0 && pg < p.num_pages ? (int64_t(pg) * 64 + (s & 63)) * p.Hkv + g : -1;
    }
    float x = 0.f, v[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      float kx = 0.f, vx = 0.f;
      if (at >= 0) {
        const int64_t i = at * D + lane * E + e;
        if constexpr (EIGHT) {
          kx = codes ? code_value(P.c.k[i]) * power(k_exp(exps)) : __bfloat162float(p.k[i]);
          vx = codes ? code_value(P.c.v[i]) * power(v_exp(exps)) : __bfloat162float(p.v[i]);
        } else {
          kx = __bfloat162float(p.k[i]);
          vx = __bfloat162float(p.v[i]);
        }
      }
      x += q[e] * kx;
      v[e] = vx;
    }
#pragma unroll
    for (int k = 16; k > 0; k >>= 1) x += __shfl_xor_sync(0xffffffffu, x, k);
    x *= p.scale_log2;
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

// Does this thread's row of O hold an infinity or a NaN? By a whole warp.
template <int D>
__device__ __noinline__ bool overflowed(uint32_t o_at) {
  uint32_t odd = 0;
#pragma unroll 1
  for (int c = 0; c < D / 32; ++c) {
    uint32_t ov[32];
    tc::tmem_ld32(o_at + c * 32, ov);
    tc::tmem_wait_ld();
#pragma unroll
    for (int e = 0; e < 32; ++e) odd |= uint32_t((ov[e] & 0x7f800000u) == 0x7f800000u);
  }
  return odd != 0u;
}

template <int D, bool PAIR, bool EIGHT, bool CLUSTER>
__global__ void __launch_bounds__(Cfg<D, PAIR, EIGHT>::THREADS, 1) window_tc_kernel(const __grid_constant__ ParamsOf<EIGHT> P) {
  using C = Cfg<D, PAIR, EIGHT>;
  using Pos = Place<C::NST>;
  const WinParams &p = P.p;
  constexpr int NST = C::NST, NR = C::NR;
  extern __shared__ uint8_t smem_raw[];
  uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  __shared__ __align__(8) uint64_t bar_full[NST], bar_empty[NST], bar_ready[NST];
  __shared__ __align__(8) uint64_t bar_qf[2], bar_qe[2], bar_s[2], bar_r[2], bar_h[2], bar_p[2], bar_o[2], bar_scan[SEEN], bar_drain[2], bar_never;
  __shared__ __align__(8) uint64_t bar_land[EIGHT ? NST : 1];  // EIGHT: the copies into a stage have landed
  __shared__ uint32_t s_exp[EIGHT ? NST : 1][2];               // and the powers of its pages
  __shared__ uint32_t s_tmem;
  __shared__ int s_abort, s_zero, s_dirty[SEEN];
  __shared__ int64_t s_beat;
  __shared__ uint8_t s_order[EIGHT && PAIR ? MAX_RANKED : 1];
  __shared__ int s_first, s_cut;  // CLUSTER: does this CTA have tiles of B; where A is cut, 0: not
  __shared__ uint32_t s_other;    // of the other CTA, 1: gave up, 2: done again row by row
  __shared__ int8_t s_par[8][64];
  __shared__ Slot s_slot[8];
  // !PAIR: (m, l) of the slots' parts, and what the rows are (EIGHT: where Q was, once all is done)
  struct RowDesc {
    int off, t;
    unsigned long long anc;
  };
  __shared__ float2 s_ml[2][PAIR || EIGHT ? 1 : ROWS];
  __shared__ RowDesc s_row[PAIR || EIGHT ? 1 : ROWS];

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t base = smem_u32(smem);
  auto q_s = [&](int w) { return base + uint32_t(PAIR ? w : 0) * C::Q_BYTES; };
  const uint32_t ring = base + C::NQ * C::Q_BYTES, land0 = smem_u32(bar_land), codes = C::IN_PLACE ? ring : ring + uint32_t(NST) * C::STAGE;
  const uint32_t full0 = smem_u32(bar_full), empty0 = smem_u32(bar_empty), ready0 = smem_u32(bar_ready);
  const uint32_t qf0 = smem_u32(bar_qf), qe0 = smem_u32(bar_qe), s0 = smem_u32(bar_s), r0 = smem_u32(bar_r), h0 = smem_u32(bar_h), p0 = smem_u32(bar_p),
                 o0 = smem_u32(bar_o), scan0 = smem_u32(bar_scan), drain0 = smem_u32(bar_drain), never = smem_u32(&bar_never);
  if (warp == TMA_WARP) {
    if (lane < NST) {
      tc::mbar_init(full0 + 8 * lane, EIGHT ? CODE_WARPS : 1);
      if constexpr (EIGHT) tc::mbar_init(land0 + 8 * lane, 1);
      tc::mbar_init(ready0 + 8 * lane, 1);  // the scan
      tc::mbar_init(empty0 + 8 * lane, 3);  // both slots, and the scan
    }
    if (lane < SEEN) {
      s_dirty[lane] = 0;
      tc::mbar_init(scan0 + 8 * lane, 1);
    }
    if (lane >= 16 && lane < 18) {
      const int w = lane - 16;
      tc::mbar_init(qf0 + 8 * w, 1);
      tc::mbar_init(qe0 + 8 * w, 1);
      tc::mbar_init(s0 + 8 * w, 1);
      tc::mbar_init(r0 + 8 * w, 128);
      tc::mbar_init(h0 + 8 * w, 128);
      tc::mbar_init(p0 + 8 * w, 128);
      tc::mbar_init(o0 + 8 * w, 1);
      tc::mbar_init(drain0 + 8 * w, 1);
    }
    if (lane == 18) {
      tc::mbar_init(never, 1);  // nothing arrives on it
      s_abort = s_zero = 0;
      s_beat = 0;
    }
    tc::fence_barrier_init();
    if (lane == 0) {
      tc::prefetch_tmap(&P.tmap_q);
      tc::prefetch_tmap(&P.tmap_k);
      tc::prefetch_tmap(&P.tmap_v);
      if constexpr (EIGHT) {
        tc::prefetch_tmap(&P.tmap_k8);
        tc::prefetch_tmap(&P.tmap_v8);
      }
    }
  }
  after_previous();  // (ahead of tensor memory too: the kernel before may still be about to take it)
  if (warp == MMA_WARP) {
    tc::tmem_alloc(smem_u32(&s_tmem), TMEM_COLS);
    tc::tmem_relinquish();
  }
  if constexpr (EIGHT && PAIR) {
    if (P.ranked) {
      int *tiles = reinterpret_cast<int *>(smem + C::NQ * C::Q_BYTES);
      rank_items(P, tiles, s_order);
      if constexpr (CLUSTER) {
        __syncthreads();
        if (tid == 0) {
          const int n = gridDim.x >> 1, a = blockIdx.x >> 1, b = 2 * n - 1 - a;
          const int na = tiles[s_order[P.hkv.div(a)]], nb = b < P.items ? tiles[s_order[P.hkv.div(b)]] : 0;
          const int cut = (na + nb + (nb > 0 ? CHANGE : 0) + 1) / 2;
          s_cut = na - cut >= LEAST ? cut : 0;
          s_first = nb;
        }
      }
    }
  }
  // (block, sequence) and KV head of item x
  auto place = [&](int x, int &turn, int &b, int &g) {
    if constexpr (EIGHT && PAIR) {
      const int e = P.hkv.div(x), i = P.ranked ? s_order[e] : e;
      turn = P.seqs.div(i);
      b = i - turn * p.B;
      g = x - e * p.Hkv;
    } else {
      turn = P.heads.div(x);
      const int bg = x - turn * int(P.heads.d);
      b = P.hkv.div(bg);
      g = bg - b * p.Hkv;
    }
  };
  // Without PAIR the item is known: its lengths and parents are on their way early.
  Lens lens{0, 0, 0};
  int early[2] = {-1, -1};
  if constexpr (!PAIR) {
    int turn, b, g;
    place(P.nsplit.div(int(blockIdx.x)), turn, b, g);
    lens = lens_of<EIGHT>(P, b);
    if (p.parent != nullptr && warp < 8) {
#pragma unroll
      for (int k = 0; k < 2; ++k)
        if (lane + 32 * k < p.T_max) early[k] = p.parent[int64_t(b) * p.T_max + lane + 32 * k];
    }
  }
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  const uint32_t tmem = s_tmem;
  volatile int *abort_flag = &s_abort;
  auto give_up = [&]() {
    if (*abort_flag == 0) {
      *abort_flag = 1;
      flag(p.status, DREAMS_DATA_TIMEOUT);
    }
  };
  auto wait = [&](uint32_t bar, uint32_t parity) { return long_wait(bar, parity & 1u, abort_flag, &s_beat, P.wait_ns); };

  // The items of this CTA; without PAIR it has one, shared by a cluster.
  const int nsplit = PAIR ? 1 : p.nsplit;
  int x_next = CLUSTER ? int(blockIdx.x & 1) ^ 1 : PAIR ? int(blockIdx.x) : P.nsplit.div(int(blockIdx.x));
  const int split = CLUSTER ? int(blockIdx.x & 1) : PAIR ? 0 : int(blockIdx.x) - x_next * nsplit;
  // the next item with work, and the tiles [j0, j1) of it that are this CTA's
  auto next_item = [&](Item &it, int &j0, int &j1, bool report) {
    if constexpr (CLUSTER) {  // x_next: 0 B, 1 A, 2 nothing
      while (x_next < 2) {
        const int n = gridDim.x >> 1, a = blockIdx.x >> 1, x = x_next == 1 ? a : 2 * n - 1 - a;
        const bool second = x_next++ == 1 && split == 1;
        if (x >= P.items || (second && s_cut == 0)) continue;
        int turn;
        place(x, turn, it.b, it.g);
        load_item<PAIR, EIGHT>(P, P.nblk - 1 - turn, it, report && !second, nullptr);
        j0 = second ? s_cut : 0;
        j1 = x == a && !second && s_cut > 0 ? s_cut : it.n;
        if (it.nb > 0 && j0 < j1) return true;
      }
    } else {
      while (x_next < P.items) {
        // the last blocks first (they have the most keys), all heads of a block together
        int turn;
        place(x_next, turn, it.b, it.g);
        load_item<PAIR, EIGHT>(P, P.nblk - 1 - turn, it, report, PAIR ? nullptr : &lens);
        if constexpr (EIGHT && PAIR) {
          // CTAs take items in order, then in reverse, and so on: who had the longest of a
          // round has the shortest of the next
          const int n = gridDim.x, of = x_next / n + 1;
          x_next = of * n + ((of & 1) ? n - 1 - int(blockIdx.x) : int(blockIdx.x));
        } else {
          x_next += PAIR ? int(gridDim.x) : P.items;
        }
        if (PAIR) {
          j0 = 0;
          j1 = it.n;
        } else {
          const Splits parts(it.n, P.nsplit);
          j0 = parts.first(split);
          j1 = parts.first(split + 1);
        }
        if (it.nb > 0 && j0 < j1) return true;
      }
    }
    return false;
  };

  // CLUSTER, and EIGHT without PAIR: this thread's row at the item's end
  Row kept{-1, 0ull};
  int kept_t = 0;
  float2 kept_ml = make_float2(-INFINITY, 0.f);
  if (warp < 8) {
    // ---------------- softmax warpgroup w: the rows of slot w
    // What an item is lies in shared memory, one copy per warp, and is read where
    // needed.
    const int w = warp >> 2;
    const int row = 32 * (warp & 3) + lane;
    const uint32_t tl = tmem + (uint32_t(32 * (warp & 3)) << 16) + 256u * w;
    const bool lead = (warp & 3) == 0 && lane == 0;
    volatile Slot *sp = &s_slot[warp];
    uint32_t sc = 0, oc = 0;  // S tiles and finished O of this slot so far
    Pos pos{0, 0};                    // K of the current tile
    bool ok = true;
    int seq = 0;
    while (ok) {
      int j, jend, gap, to;  // tiles j .. jend-1 but for [gap, to), which only the other slot reads
      int wfrom, wto;        // tiles that all rows see whole
      bool live;             // does this warp have rows?
      bool whole = true;     // are all of the item's tiles this CTA's?
      int ahead;             // stages from here to the next item
      {
        Item it;
        int j0, j1;
        if (!next_item(it, j0, j1, false)) break;
        const int blk = PAIR ? w : 0;
        const bool here = !PAIR || w < it.nb;
        const int t0 = blk ? it.t01 : it.t00, rows_blk = here ? ((blk ? it.tl1 : it.tl0) - t0 + 1) * p.G : 0;
        live = 32 * (warp & 3) < rows_blk;
        const Whole wh = whole_tiles(p, it, blk);
        wfrom = wh.from;
        wto = wh.to;
        j = j0;
        jend = j1;
        if (CLUSTER) whole = j1 - j0 == it.n;
        gap = to = INT_MAX;
        if (PAIR) {
          if (!here) jend = j;
          else if (w == 0) jend = CLUSTER ? ::min(j1, it.e0) : it.e0;
          else if (it.a1 > it.ns) {
            gap = it.ns;
            to = it.a1;
          }
          if (CLUSTER) {
            to = ::min(to, j1);
            if (here && j >= gap) j = ::max(j, to);
          } else if (here && j >= gap) {
            j = to;
          }
        } else {
          j = ::min(j1, j0 + w);
        }
        pos.move(2 * (j - j0));
        ahead = 2 * (j1 - j);
        __syncwarp();  // the last item's readers are done
        if (lane == 0) {
          sp->L = it.L;
          sp->view.first = it.column(it.L - p.window + 1);
          sp->view.lowest = it.column(it.lo);
          sp->view.fresh = it.column(it.L);
          sp->view.sinks = it.nsp > 0 ? it.S1 : p.sinks;
          sp->cols = it.column(it.hi);
          sp->t0 = t0;
          sp->rows = rows_blk;
          sp->b = it.b;
          sp->g = it.g;
        }
        int bad = 0;
        if (p.parent != nullptr) {
          for (int i = lane; i < it.T; i += 32) {
            const int q = PAIR ? p.parent[int64_t(it.b) * p.T_max + i] : i < 32 ? early[0] : early[1];
            s_par[warp][i] = int8_t(q);  // (a bad one is not used)
            bad |= i == 0 ? q != -1 : (q < 0 || q >= i);
          }
          bad = __any_sync(0xffffffffu, bad);
          if (bad && lead && w == 0 && it.g == 0 && (CLUSTER ? j0 : split) == 0) flag(p.status, DREAMS_DATA_BAD_PARENT);
        }
        if (lane == 0) sp->bad = bad;
        __syncwarp();
      }
      const bool any = j < jend;
      // this thread's row, and what it sees
      Row r;
      int t = 0;
      {
        const int t0 = sp->t0;
        t = row < sp->rows ? t0 + P.g.div(row) : t0;
        r.off = t;
        r.anc = 0ull;
        if (p.parent != nullptr && row < sp->rows && sp->bad == 0) r.anc = tree_row(p, s_par[warp], sp->L, t, r.off);
      }
      float m_ref = -INFINITY, l = 0.f;
      bool unset = true;  // does a row of this warp lack its reference?
      int v1 = -1;        // V stage of the last tile
      const uint64_t scale2 = f32x2(p.scale_log2, p.scale_log2);
      while (j < jend) {
        ok = wait(s0 + 8 * w, sc);
        if (!__all_sync(0xffffffffu, ok)) {
          ok = false;
          break;
        }
        ++sc;
        tc::fence_after_sync();
        // This slot's MMAs up to this S are done: the lead thread gives back K of this
        // tile, V of the one before (P over S: its P V is), and Q after the last.
        const Pos vp = pos.plus(1);
        int nj = j + (PAIR ? 1 : 2);
        if (PAIR && nj == gap) nj = to;
        arrive_if(empty0 + 8 * pos.s, lead);
        if (!C::BESIDE) arrive_if(empty0 + 8 * v1, lead && v1 >= 0);
        if (PAIR) arrive_if(qe0 + 8 * w, lead && nj >= jend);
        const int v0 = v1;  // V stage of the tile before
        v1 = vp.s;

        const bool full = j >= wfrom && j < wto;
        int nc = KT;
        uint32_t mask[4] = {~0u, ~0u, ~0u, ~0u};
        uint32_t none = 0, part = 0;  // groups of 32 columns that no row of the warp sees; that some see in part
        if (__builtin_expect(!full, 0)) {
          View v;
          asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.first), "=r"(v.lowest), "=r"(v.fresh), "=r"(v.sinks) : "r"(smem_u32(&s_slot[warp].view)));
          nc = ::min(KT, (sp->cols - j * KT + 31) & ~31);
          const bool tree = p.parent != nullptr;
          const int from = ::max(r.off + v.first, v.lowest), to = tree ? v.fresh : v.fresh + r.off + 1, sinks = ::min(v.sinks, to);
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const int col = j * KT + 32 * c;
            uint32_t m = low_bits(sinks - col) | (low_bits(to - col) & ~low_bits(from - col));
            if (tree) {
              const int sh = col - v.fresh;
              m |= (sh >= 64 || sh <= -32) ? 0u : (sh >= 0 ? uint32_t(r.anc >> sh) : uint32_t(r.anc << (-sh)));
            }
            mask[c] = m;
            none |= uint32_t(!__any_sync(0xffffffffu, m != 0u)) << c;
            part |= uint32_t(!__all_sync(0xffffffffu, m == ~0u)) << c;
          }
        }
        if (__builtin_expect(unset, 0)) {
          // references: the maximum of the first 32 columns that hold a key of theirs,
          // for rows that have none
          if (live) {
#pragma unroll 1
            for (int c = 0; 32 * c < nc && unset; ++c) {
              const uint32_t m = c == 0 ? mask[0] : c == 1 ? mask[1] : c == 2 ? mask[2] : mask[3];
              if ((none >> c) & 1u) continue;
              uint32_t u[32];
              float mx = -INFINITY;
              tc::tmem_ld32(tl + 32 * c, u);
              tc::tmem_wait_ld();
#pragma unroll
              for (int e = 0; e < 32; ++e) mx = fmaxf(mx, ((m >> e) & 1u) ? __uint_as_float(u[e]) : -INFINITY);
              if (m_ref == -INFINITY) m_ref = mx * p.scale_log2;  // scale > 0
              unset = __any_sync(0xffffffffu, row < sp->rows && m_ref == -INFINITY);
            }
          } else {
            unset = false;
          }
        }
        const float nmu = m_ref == -INFINITY ? 0.f : -m_ref;
        const uint64_t nmu2 = f32x2(nmu, nmu);
        uint64_t acc2[2] = {f32x2(0.f, 0.f), f32x2(0.f, 0.f)};
        // P of 64 keys at a time, as bf16 over the first half of S, or beside it
#pragma unroll 1
        for (int hh = 0; hh < 2; ++hh) {
          uint32_t u[64];
          const bool some = live && ((none >> (2 * hh)) & 3u) != 3u;  // (columns from nc on are none's)
          if (some) {
            tc::tmem_ld32(tl + 64 * hh, *reinterpret_cast<uint32_t(*)[32]>(&u[0]));
            tc::tmem_ld32(tl + 64 * hh + 32, *reinterpret_cast<uint32_t(*)[32]>(&u[32]));
            tc::tmem_wait_ld();
            if (__builtin_expect((part >> (2 * hh)) & 3u, 0)) {
              const uint32_t m0 = hh ? mask[2] : mask[0], m1 = hh ? mask[3] : mask[1];
#pragma unroll
              for (int e = 0; e < 32; ++e) {
                if (!((m0 >> e) & 1u)) u[e] = 0xff800000u;
                if (!((m1 >> e) & 1u)) u[32 + e] = 0xff800000u;
              }
            }
          }
          if (C::BESIDE && hh == 1) {
            tc::fence_before_sync();
            tc::mbar_arrive(r0 + 8 * w);  // S may be overwritten
          }
          if (C::BESIDE && hh == 0 && v0 >= 0) {
            // P may be overwritten once the P V before is done; and its V goes back
            ok = wait(o0 + 8 * w, oc);
            if (!__all_sync(0xffffffffu, ok)) {
              ok = false;
              break;
            }
            ++oc;
            tc::fence_after_sync();
            arrive_if(empty0 + 8 * v0, lead);
          }
          if (some) {
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              uint32_t pk[16];
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                float e0, e1;
                f32x2_split(ffma2(f32x2(__uint_as_float(u[32 * c + 2 * i]), __uint_as_float(u[32 * c + 2 * i + 1])), scale2, nmu2), e0, e1);
                const float a = tc::ex2(e0), b = tc::ex2(e1);
                acc2[i & 1] = fadd2(acc2[i & 1], f32x2(a, b));
                pk[i] = pack_bf16x2(a, b);
              }
              tc::tmem_st16(tl + C::P_COL + 32 * hh + 16 * c, pk);
            }
            tc::tmem_wait_st();
          } else if (live && 64 * hh < nc) {
            const uint32_t zero[16] = {};
            tc::tmem_st16(tl + C::P_COL + 32 * hh, zero);
            tc::tmem_st16(tl + C::P_COL + 32 * hh + 16, zero);
            tc::tmem_wait_st();
          }
          tc::fence_before_sync();
          tc::mbar_arrive((hh == 0 ? h0 : p0) + 8 * w);
        }
        if (!ok) break;
        {
          float a0, a1, b0, b1;
          f32x2_split(acc2[0], a0, a1);
          f32x2_split(acc2[1], b0, b1);
          l += (a0 + a1) + (b0 + b1);
        }
        pos = pos.plus(2);
        if (!PAIR) pos = pos.plus(2);
        else if (nj != j + 1) {
          pos.move(2 * (nj - j - 1));
          if (!C::BESIDE && (!CLUSTER || nj < jend)) v1 = -1;  // (before a gap the issuer's commit gives V back)
        }
        ahead -= 2 * (nj - j);
        j = nj;
      }
      if (ok && any) {
        ok = __all_sync(0xffffffffu, wait(o0 + 8 * w, oc));  // all MMAs of the slot are done
        ++oc;
        tc::fence_after_sync();
        if (ok) arrive_if(empty0 + 8 * v1, lead);
        ok = ok && __all_sync(0xffffffffu, wait(scan0 + 8 * (seq % SEEN), uint32_t(seq / SEEN)));
      }
      if (!ok) break;
      if (PAIR) pos.move(ahead);
      const bool dirty = *reinterpret_cast<volatile int *>(&s_dirty[seq % SEEN]) != 0;  // (of use where `any`)
      ++seq;

      const bool real = row < sp->rows, tree_ok = sp->bad == 0;
      if (CLUSTER && !whole) {
        kept = Row{tree_ok ? r.off : -1, r.anc};
        kept_t = t;
        if (any && live) kept_ml = make_float2(m_ref, l);
      } else if constexpr (PAIR) {
        const int h = sp->g * p.G + row - (t - sp->t0) * p.G;
        uint32_t again = __ballot_sync(0xffffffffu, any && real && (dirty || l > SAFE_SUM));
        if (__builtin_expect(again != 0u, 0)) {
          const bool odd = overflowed<D>(tl + C::O_COL);
          again &= __ballot_sync(0xffffffffu, dirty || l > MOST_SUM || odd);
        }
        if (any && tree_ok) {
          const float inv = 1.f / l;
          const int64_t orow = (int64_t(sp->b) * p.T_max + t) * p.Hq + h;
          if (live) {
            const bool write = real && !((again >> lane) & 1u), wide = (reinterpret_cast<uintptr_t>(p.out) & 31u) == 0;
            uint4 *dst = reinterpret_cast<uint4 *>(p.out + orow * D);
#pragma unroll 1
            for (int c = 0; c < D / 32; ++c) {
              uint32_t ov[32];
              tc::tmem_ld32(tl + C::O_COL + c * 32, ov);
              tc::tmem_wait_ld();
              uint32_t pk[16];
#pragma unroll
              for (int e = 0; e < 16; ++e) pk[e] = pack_bf16x2(__uint_as_float(ov[2 * e]) * inv, __uint_as_float(ov[2 * e + 1]) * inv);
              if (write && wide) {
                st_global_v8(dst + 4 * c, pk);
                st_global_v8(dst + 4 * c + 2, pk + 8);
              } else if (write) {
#pragma unroll
                for (int e = 0; e < 4; ++e) dst[4 * c + e] = make_uint4(pk[4 * e], pk[4 * e + 1], pk[4 * e + 2], pk[4 * e + 3]);
              }
            }
            if (real && !((again >> lane) & 1u) && p.lse != nullptr) p.lse[orow] = (m_ref + log2f(l)) * LN2;
          }
        }
        if (__builtin_expect(again != 0u && tree_ok, 0)) {
          __syncwarp();  // the stores above come first
          for (int i = 0; i < 32; ++i) {
            const int ti = __shfl_sync(0xffffffffu, t, i), oi = __shfl_sync(0xffffffffu, r.off, i), hi = __shfl_sync(0xffffffffu, h, i);
            const unsigned long long ai = __shfl_sync(0xffffffffu, r.anc, i);
            if ((again >> i) & 1u) slow_row<D, EIGHT>(P, sp->b, sp->g, sp->L, ti, hi, oi, ai, &s_beat);
          }
        }
        tc::fence_before_sync();  // O may be overwritten once this warpgroup's next P has arrived
      } else if constexpr (EIGHT) {
        kept = Row{tree_ok ? r.off : -1, r.anc};
        kept_t = t;
        if (any && live) kept_ml = make_float2(m_ref, l);
      } else {
        // what the rows are, and the slot's (m, l), for the join below
        if (w == 0) {
          s_row[row].off = tree_ok ? r.off : -1;
          s_row[row].t = t;
          s_row[row].anc = r.anc;
        }
        s_ml[w][row] = any && live ? make_float2(m_ref, l) : make_float2(-INFINITY, 0.f);
      }
    }
    if (!ok) give_up();
  } else {
    if (warp == TMA_WARP) {
      // ---------------- producer: for each item K_0, Q, V_0, K_1, V_1, ...
      if (lane == 0) {
        Pos at{0, 0};
        bool wrapped = false, ok = true;
        int issued = 0, ktiles = 0;
        uint32_t nq[2] = {0, 0};
        Item it;
        int j0, j1;
        while (ok && next_item(it, j0, j1, CLUSTER || split == 0)) {
          const int32_t *row = p.table != nullptr ? p.table + int64_t(it.b) * p.P : nullptr;
          auto fetch = [&](int j, int h) {
            if (j >= j1 || 2 * j + h >= it.np) return 0;
            const int pi = it.slot0(2 * j + h) >> 6;
            if constexpr (EIGHT) {
              if (it.codes(2 * j + h)) return P.c.table[int64_t(it.b) * P.c.P + pi];
            }
            if (row == nullptr) return 0;
            return pi < p.P ? row[pi] : -1;
          };
          auto powers = [&](int j, int h, int pg) -> uint32_t {
            if constexpr (EIGHT) {
              if (j < j1 && it.codes(2 * j + h) && pg >= 0 && pg < P.c.num_pages) return P.c.exps[int64_t(pg) * p.Hkv + it.g];
            }
            return 0u;
          };
          int pg0 = fetch(j0, 0), pg1 = fetch(j0, 1);
          for (int j = j0; j < j1 && ok; ++j) {
            const int halves = 2 * j + 1 < it.np ? 2 : 1, ha = it.slot0(2 * j), hb = it.slot0(2 * j + 1);
            // tensor-map coordinate (dim 3) of a half: outside the map (zeros) where the
            // page is missing
            const bool c0 = EIGHT && it.codes(2 * j), c1 = EIGHT && it.codes(2 * j + 1);
            auto coord = [&](int h, int pg) {
              if constexpr (EIGHT) {
                if (h == 0 ? c0 : c1) {
                  if (pg >= 0 && pg < P.c.num_pages) return pg;
                  flag(p.status, DREAMS_DATA_BAD_PAGE);
                  return P.c.num_pages;
                }
              }
              if (row == nullptr) return it.b;
              if (pg >= 0 && pg < p.num_pages) return pg;
              if (h < halves) flag(p.status, DREAMS_DATA_BAD_PAGE);
              return p.num_pages;
            };
            const int ca = coord(0, pg0), cb = coord(1, pg1), sa = row != nullptr ? 0 : ha, sb = row != nullptr ? 0 : hb;
            const uint32_t x0 = powers(j, 0, pg0), x1 = powers(j, 1, pg1);  // (waited for where they are used)
            pg0 = fetch(j + 1, 0);
            pg1 = fetch(j + 1, 1);
#pragma unroll 1
            for (int kv = 0; kv < 2 && ok; ++kv) {
              if (kv == 0 && P.stall_at >= 0 && ktiles >= P.stall_at) {
                // test hook: this copy is never issued
                tc::mbar_wait(never, 0, abort_flag, P.wait_ns);
                ok = false;
                break;
              }
              if (wrapped && !wait(empty0 + 8 * at.s, at.ph ^ 1u)) {
                ok = false;
                break;
              }
              const uint32_t st = ring + uint32_t(at.s) * C::STAGE, bar = (EIGHT ? land0 : full0) + 8 * at.s;
              const int coded = int(c0) + int(c1);
              if constexpr (EIGHT) {
                s_exp[at.s][0] = x0;
                s_exp[at.s][1] = x1;
              }
              tc::mbar_arrive_expect_tx(bar, uint32_t(NR * (halves - coded) * 8192 + coded * 64 * D));
              if constexpr (EIGHT) {
                const uint32_t to = codes + uint32_t(at.s) * C::CODES;
                const CUtensorMap *map = kv == 0 ? &P.tmap_k8 : &P.tmap_v8;
                if (c0) tc::tma_load_4d(to, map, bar, 0, it.g, 0, ca);
                if (c1) tc::tma_load_4d(to + C::HALF, map, bar, 0, it.g, 0, cb);
              }
              const CUtensorMap *map = kv == 0 ? &P.tmap_k : &P.tmap_v;
#pragma unroll
              for (int r = 0; r < NR; ++r) {
                if (!c0) tc::tma_load_4d(st + r * C::KV_REGION, map, bar, r * 64, it.g, sa, ca);
                if (halves == 2 && !c1) tc::tma_load_4d(st + r * C::KV_REGION + 8192, map, bar, r * 64, it.g, sb, cb);
              }
              ++issued;
              at = at.plus(1);
              wrapped |= at.s == 0;
              if (kv == 1) break;
              ++ktiles;
              if (j == j0) {  // the item's Q, once the last item's is done with
#pragma unroll
                for (int w = 0; w < C::NQ; ++w) {
                  if (w >= it.nb || !ok) continue;
                  if (nq[w] > 0 && !wait(qe0 + 8 * w, nq[w] - 1)) {
                    ok = false;
                    continue;
                  }
                  ++nq[w];
                  tc::mbar_arrive_expect_tx(qf0 + 8 * w, uint32_t(NR * p.G * P.TB * 128));
#pragma unroll
                  for (int r = 0; r < NR; ++r)
                    tc::tma_load_5d(q_s(w) + r * C::Q_REGION, &P.tmap_q, qf0 + 8 * w, r * 64, 0, it.g, w ? it.t01 : it.t00, it.b);
                }
              }
            }
          }
        }
        if (!ok) give_up();
        // no copy may still be landing when the CTA ends
        for (int i = ::max(0, issued - NST); i < issued; ++i) tc::mbar_wait((EIGHT ? land0 : full0) + 8 * (i % NST), (i / NST) & 1, &s_zero);
        for (int w = 0; w < C::NQ; ++w)
          if (nq[w] > 0) tc::mbar_wait(qf0 + 8 * w, (nq[w] - 1) & 1u, &s_zero);
      }
    } else if (warp < SCAN_WARP) {
      // ---------------- MMA issuers, one for each slot: the tensor pipe takes their
      // instructions as they come, so one's waits run under the other's MMAs
      if (lane == 0) {
        const int w = warp - MMA_WARP;
        // low words of the operands' descriptors: address / 16 (of 18 bits: in a
        // cluster the bits above say which CTA), leading-dimension offset / 16
        const uint32_t ring16 = (ring & 0x3FFFFu) >> 4;
        const uint32_t q_lo = ((q_s(w) & 0x3FFFFu) >> 4) | (1u << 16), k_lo = ring16 | (1u << 16), v_lo = ring16 | ((C::KV_REGION >> 4) << 16);
        const uint32_t s_col = tmem + 256u * w, p_col = s_col + C::P_COL, o_col = s_col + C::O_COL;
        constexpr uint32_t IDESC_QK = tc::idesc_bf16_f32(ROWS, 0, false);
        constexpr uint32_t IDESC_PV = tc::idesc_bf16_f32(ROWS, D, true);
        // S = Q K^T over the first nc keys of a stage
        auto qk = [&](int st, int nc) {
          const uint32_t idesc = IDESC_QK | (uint32_t(nc >> 3) << 17);
          const uint32_t k = k_lo + uint32_t(st) * (C::STAGE >> 4);
#pragma unroll
          for (int i = 0; i < D / 16; ++i) {
            const uint32_t off = (i & 3) << 5;
            mma_ss(s_col, q_lo + (((i >> 2) * C::Q_REGION + off) >> 4), k + (((i >> 2) * C::KV_REGION + off) >> 4), idesc, i > 0 ? 1u : 0u);
          }
          tc::mma_commit(s0 + 8 * w);
        };
        bool ok = true;
        Pos at{0, 0};                      // K of the item's first tile
        uint32_t pc = 0, qc = 0;           // P tiles and Q blocks so far
        Item it;
        int j0, j1;
        while (ok && next_item(it, j0, j1, false)) {
          const bool here = !PAIR || w < it.nb;
          auto next_of = [&](int j) {
            int k = j + (PAIR ? 1 : 2);
            if (!PAIR) return ::min(j1, k);
            if (w == 0) return k < (CLUSTER ? ::min(j1, it.e0) : it.e0) ? k : j1;
            const int to = k >= it.ns ? ::max(k, it.a1) : k;
            return CLUSTER ? ::min(j1, to) : to;
          };
          // tiles [a, e) are the other slot's: this one gives them back unread
          Pos pos = at;  // K of the first tile not dealt with
          auto skip = [&](int a, int e) {
#pragma unroll 1
            for (int x = 2 * a; x < 2 * e && ok; ++x) {
              ok = wait(full0 + 8 * pos.s, pos.ph);
              if (ok) tc::mbar_arrive(empty0 + 8 * pos.s);
              pos = pos.plus(1);
            }
          };
          int j = !here ? j1 : PAIR ? next_of(j0 - 1) : ::min(j1, j0 + w);
          skip(j0, j);
          Pos kp = pos;
          if (ok && j < j1) {
            ok = wait(qf0 + 8 * (PAIR ? w : 0), qc) && wait(full0 + 8 * kp.s, kp.ph);
            ++qc;
            if (!ok) break;
            tc::fence_after_sync();
            qk(kp.s, it.ncols(j));
          }
          bool first = true;
          while (j < j1 && ok) {
            const int nj = next_of(j), nc = it.ncols(j), nnc = nj < j1 ? it.ncols(nj) : 0;
            const Pos vp = kp.plus(1);
            pos = kp.plus(2);
            // what the copies bring is waited for ahead of P
            ok = wait((it.cut(j) ? ready0 : full0) + 8 * vp.s, vp.ph);
            if ((C::BESIDE || PAIR) && ok && nj < j1) {
              skip(j + 1, nj);
              ok = ok && wait(full0 + 8 * pos.s, pos.ph);
            }
            ok = ok && wait(h0 + 8 * w, pc);
            if (!ok) break;
            // O (+)= P V, P in two halves of 64 keys
            const uint32_t v = v_lo + uint32_t(vp.s) * (C::STAGE >> 4);
            tc::fence_after_sync();
#pragma unroll
            for (int k = 0; k < 4; ++k)
              if (16 * k < nc) mma_ts(o_col, p_col + 8 * k, v + k * 128, IDESC_PV, (k > 0 || !first) ? 1u : 0u);
            if (C::BESIDE) {
              // S has been read: the next one
              ok = wait(r0 + 8 * w, pc);
              if (!ok) break;
              tc::fence_after_sync();
              if (nj < j1) qk(pos.s, nnc);
            }
            ok = wait(p0 + 8 * w, pc);
            if (!ok) break;
            tc::fence_after_sync();
#pragma unroll
            for (int k = 4; k < 8; ++k)
              if (16 * k < nc) mma_ts(o_col, p_col + 8 * k, v + k * 128, IDESC_PV, 1u);
            ++pc;
            first = false;
            if (C::BESIDE || nj >= j1) tc::mma_commit(o0 + 8 * w);
            if (!C::BESIDE && nj < j1) {
              if (PAIR && nj != j + 1) tc::mma_commit(empty0 + 8 * vp.s);  // before a gap: no S announces that this V is read
              if (!PAIR) {
                skip(j + 1, nj);
                ok = ok && wait(full0 + 8 * pos.s, pos.ph);
                if (!ok) break;
                tc::fence_after_sync();
              }
              qk(pos.s, nnc);
            }
            if (nj >= j1) skip(j + 1, j1);
            kp = pos;
            j = nj;
          }
          at.move(2 * (j1 - j0));
        }
        if (!ok) give_up();
        tc::mma_commit(drain0 + 8 * w);
        tc::mbar_wait(drain0 + 8 * w, 0, &s_zero);
      }
    } else if (warp >= CODE_WARP) {
      if constexpr (EIGHT) {
        // ---------------- codes to bf16: each warp 16 rows of a page. A code times its page's
        // power is exact in bf16, so what follows does not know of codes.
        // A lane's 16 codes of a row are two runs of 8, each 16 bytes of a row's bf16; which of
        // them is first differs between lanes, so that no two of eight meet in a bank.
        constexpr int CH = D / 16;
        const int cw = warp - CODE_WARP, ch = lane % CH, lr = lane / CH, part = D == 128 ? ((ch >> 2) ^ (lr & 1)) : 0;
        const uint32_t mine = codes + uint32_t((16 * cw + lr) * D + ch * 16 + part * 8), flip = part != 0 ? uint32_t(-8) : 8u;
        const uint32_t put = ring + 2048u * cw + (ch >> 2) * C::KV_REGION + lr * 128 + (uint32_t((2 * (ch & 3) + part) ^ lr) << 4);
        Pos at{0, 0};
        bool ok = true;
        Item it;
        int j0, j1;
        while (ok && next_item(it, j0, j1, false)) {
          for (int j = j0; j < j1 && ok; ++j) {
            const bool c0 = it.codes(2 * j), c1 = it.codes(2 * j + 1);
#pragma unroll 1
            for (int kv = 0; kv < 2; ++kv) {
              ok = __all_sync(0xffffffffu, wait(land0 + 8 * at.s, at.ph));
              if (!ok) break;
              if (c0) {  // (the first half is in 8 bits where the second is)
                const uint32_t x0 = *reinterpret_cast<volatile uint32_t *>(&s_exp[at.s][0]), x1 = *reinterpret_cast<volatile uint32_t *>(&s_exp[at.s][1]);
                const int e0 = kv == 0 ? k_exp(x0) : v_exp(x0), e1 = kv == 0 ? k_exp(x1) : v_exp(x1);
                const bool large = (e0 > 7 && e0 != DREAMS_KV8_NOT_FINITE) || (e1 > 7 && e1 != DREAMS_KV8_NOT_FINITE);
                const uint32_t from = mine + uint32_t(at.s) * C::CODES, to = put + uint32_t(at.s) * C::STAGE;
                if (__builtin_expect(large || !c1, 0)) {
                  widen_rare<D>(from, to, e0, flip);
                  if (c1) widen_rare<D>(from + C::HALF, to + 8192, e1, flip);
                } else {
                  widen<D, C::HALF>(from, to, e0, e1, flip);
                }
                tc::fence_proxy_async_smem();
              }
              __syncwarp();
              if (lane == 0) tc::mbar_arrive(full0 + 8 * at.s);
              at = at.plus(1);
            }
          }
        }
        if (!ok) give_up();
      }
    } else {
      // ---------------- the scan: where rows see a tile in part, an infinity or a
      // NaN in V would reach the others (0 x inf); such items are done again row by row
      Pos at{0, 0};
      bool ok = true;
      Item it;
      int j0, j1, seq = 0;
      while (ok && next_item(it, j0, j1, false)) {
        const Whole w0 = whole_tiles(p, it, 0), w1 = whole_tiles(p, it, 1);
        uint32_t acc = 0;  // sums of 0 x V: zero, or NaN
        for (int j = j0; j < j1 && ok; ++j) {
          const bool look = (it.need0(j) && !w0(j)) || (it.need1(j) && !w1(j));
#pragma unroll 1
          for (int kv = 0; kv < 2; ++kv) {
            ok = __all_sync(0xffffffffu, wait(full0 + 8 * at.s, at.ph));
            if (!ok) break;
            const uint32_t st = ring + uint32_t(at.s) * C::STAGE + ((lane & 7) << 4);
            const int halves = 2 * j + 1 < it.np ? 2 : 1;
            if (kv == 1) {
              // lanes along a row's 128 bytes, four rows at a time; slots that no row
              // sees may hold any bits: their V rows become zeros
              bool cut = false;
              for (int h = 0; h < halves; ++h) {
                const int b0 = it.beg(2 * j + h), e0 = it.end(2 * j + h);
                cut |= b0 > 0 || e0 < 64;
#pragma unroll 1
                for (int z = lane >> 3; z < b0 + 64 - e0; z += 4) {
                  const int rr = 64 * h + (z < b0 ? z : e0 + z - b0);
#pragma unroll
                  for (int r = 0; r < NR; ++r)
                    asm volatile("st.shared.v4.b32 [%0], {%1,%1,%1,%1};" ::"r"(st + r * C::KV_REGION + rr * 128), "r"(0u) : "memory");
                }
              }
              if (cut) tc::fence_proxy_async_smem();
            }
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(ready0 + 8 * at.s);
            if (kv == 1 && look) {
              for (int h = 0; h < halves; ++h) {
                const int r1 = 64 * h + it.end(2 * j + h);
#pragma unroll 4
                for (int rr = 64 * h + it.beg(2 * j + h) + (lane >> 3); rr < r1; rr += 4) {
#pragma unroll
                  for (int r = 0; r < NR; ++r) {
                    uint32_t u[4];
                    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];"
                                 : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3])
                                 : "r"(st + r * C::KV_REGION + rr * 128));
#pragma unroll
                    for (int e = 0; e < 4; ++e) asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(acc) : "r"(u[e]), "r"(0u));
                  }
                }
              }
            }
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(empty0 + 8 * at.s);
            at = at.plus(1);
          }
        }
        const bool bad = __any_sync(0xffffffffu, (acc & 0x7fff7fffu) != 0u);
        if (lane == 0) {
          s_dirty[seq % SEEN] = bad;
          if (ok) tc::mbar_arrive(scan0 + 8 * (seq % SEEN));
        }
        ++seq;
      }
      if (!ok) give_up();
    }
  }

  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  if constexpr (CLUSTER) {
    // ---------------- join the two parts of A: CTA w finishes block w, whose other part is
    // pushed into its ring once both are done with theirs
    if (s_cut > 0) {
      Item it;
      int turn;
      place(blockIdx.x >> 1, turn, it.b, it.g);
      load_item<PAIR, EIGHT>(P, P.nblk - 1 - turn, it, false, nullptr);
      constexpr int CH = D / 4;  // 16-byte columns of a part's row, swizzled by the row
      float *part = reinterpret_cast<float *>(smem + C::NQ * C::Q_BYTES);
      float2 *mls = reinterpret_cast<float2 *>(part + ROWS * D);
      static_assert(size_t(NST) * C::STAGE >= ROWS * (D * 4 + sizeof(float2)), "a part fits");
      const int w = (warp >> 2) & 1, row = 32 * (warp & 3) + lane;
      const int rows = w < it.nb ? ((w ? it.tl1 : it.tl0) - (w ? it.t01 : it.t00) + 1) * p.G : 0;
      const bool live = warp < 8 && 32 * (warp & 3) < rows, mine = w == split;
      const bool dirty = s_dirty[split == 1 && s_first > 0 ? 1 : 0] != 0;
      const uint32_t tl = tmem + (uint32_t(32 * (warp & 3)) << 16) + 256u * w + C::O_COL;
      cluster_sync();
      if (tid == 0) st_cluster(mapa(smem_u32(&s_other), split ^ 1), (s_abort ? 1u : 0u) | (dirty ? 2u : 0u));
      if (live && !mine) {
        st_cluster2(mapa(smem_u32(mls + row), split ^ 1), kept_ml);
        if (__any_sync(0xffffffffu, kept_ml.y != 0.f)) {
          const uint32_t to = mapa(smem_u32(part + row * D), split ^ 1);
#pragma unroll 1
          for (int c = 0; c < D / 32; ++c) {
            uint32_t ov[32];
            tc::tmem_ld32(tl + c * 32, ov);
            tc::tmem_wait_ld();
#pragma unroll
            for (int e = 0; e < 8; ++e) st_cluster4(to + (((c * 8 + e) ^ (row & (CH - 1))) << 4), ov + 4 * e);
          }
        }
      }
      __syncwarp();
      cluster_sync();
      const uint32_t state = s_other | (s_abort ? 1u : 0u) | (dirty ? 2u : 0u);
      if (live && mine && !(state & 1u)) {
        const float2 own = kept_ml, far = mls[row];
        const bool real = row < rows && kept.off >= 0;  // (not of a malformed tree)
        const float M = fmaxf(own.x, far.x), c0 = own.y == 0.f ? 0.f : tc::ex2(own.x - M), c1 = far.y == 0.f ? 0.f : tc::ex2(far.x - M);
        const float Z = c0 * own.y + c1 * far.y;
        // columns 32 c .. 32 c + 31 of the row, both parts
        auto both = [&](int c, float (&o)[32]) {
          uint32_t ov[32];
          tc::tmem_ld32(tl + c * 32, ov);
          tc::tmem_wait_ld();
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float4 f = *reinterpret_cast<const float4 *>(part + row * D + (((c * 8 + e) ^ (row & (CH - 1))) << 2));
            const float fv[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const float a = own.y == 0.f ? 0.f : c0 * __uint_as_float(ov[4 * e + k]);  // (a part without keys may be anything)
              o[4 * e + k] = far.y == 0.f ? a : a + c1 * fv[k];
            }
          }
        };
        const bool wild = own.y > SAFE_SUM || far.y > SAFE_SUM;
        bool redo = (state & 2u) || own.y > MOST_SUM || far.y > MOST_SUM;
        if (__builtin_expect(__any_sync(0xffffffffu, wild), 0)) {
          float odd = 0.f;  // (a sum of 0 x O is zero, or NaN)
#pragma unroll 1
          for (int c = 0; c < D / 32; ++c) {
            float o[32];
            both(c, o);
#pragma unroll
            for (int e = 0; e < 32; ++e) odd += 0.f * o[e];
          }
          redo = redo || (wild && odd != 0.f);
        }
        const uint32_t again = __ballot_sync(0xffffffffu, real && redo);
        const int h = it.g * p.G + row - (kept_t - (w ? it.t01 : it.t00)) * p.G;
        const int64_t orow = (int64_t(it.b) * p.T_max + kept_t) * p.Hq + h;
        const bool write = real && !redo, wide = (reinterpret_cast<uintptr_t>(p.out) & 31u) == 0;
        const float inv = 1.f / Z;
        uint4 *dst = reinterpret_cast<uint4 *>(p.out + orow * D);
#pragma unroll 1
        for (int c = 0; c < D / 32; ++c) {
          float o[32];
          both(c, o);
          uint32_t pk[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) pk[e] = pack_bf16x2(o[2 * e] * inv, o[2 * e + 1] * inv);
          if (write && wide) {
            st_global_v8(dst + 4 * c, pk);
            st_global_v8(dst + 4 * c + 2, pk + 8);
          } else if (write) {
#pragma unroll
            for (int e = 0; e < 4; ++e) dst[4 * c + e] = make_uint4(pk[4 * e], pk[4 * e + 1], pk[4 * e + 2], pk[4 * e + 3]);
          }
        }
        if (write && p.lse != nullptr) p.lse[orow] = (M + log2f(Z)) * LN2;
        if (__builtin_expect(again != 0u, 0)) {
          for (int i = 0; i < 32; ++i) {
            const int ti = __shfl_sync(0xffffffffu, kept_t, i), oi = __shfl_sync(0xffffffffu, kept.off, i), hi = __shfl_sync(0xffffffffu, h, i);
            const unsigned long long ai = __shfl_sync(0xffffffffu, kept.anc, i);
            if ((again >> i) & 1u) slow_row<D, EIGHT>(P, it.b, it.g, it.L, ti, hi, oi, ai, &s_beat);
          }
        }
      }
      tc::fence_before_sync();
      __syncthreads();
      tc::fence_after_sync();
    }
  }
  if constexpr (!PAIR) {
    // ---------------- join the slots' and the splits' parts
    x_next = P.nsplit.div(int(blockIdx.x));
    Item it;
    int turn;
    place(x_next, turn, it.b, it.g);
    load_item<PAIR, EIGHT>(P, P.nblk - 1 - turn, it, false, &lens);
    const Splits splits(it.n, P.nsplit);
    const int m = splits.first(split + 1) - splits.first(split);
    const int rows_blk = it.nb > 0 ? (it.tl0 - it.t00 + 1) * p.G : 0;
    constexpr int CH = D / 4;  // 16-byte columns of a part's row, swizzled by the row
    float *part = reinterpret_cast<float *>(smem + C::NQ * C::Q_BYTES);
    auto *mls = EIGHT ? reinterpret_cast<float2(*)[ROWS]>(smem) : reinterpret_cast<float2(*)[ROWS]>(&s_ml[0][0]);
    RowDesc *descs = EIGHT ? reinterpret_cast<RowDesc *>(smem + 2 * ROWS * sizeof(float2)) : s_row;
    static_assert(!EIGHT || C::Q_BYTES >= ROWS * (2 * sizeof(float2) + sizeof(RowDesc)), "they fit");
    if (warp < 8) {
      const int w = warp >> 2, row = 32 * (warp & 3) + lane;
      const bool has = w < m && s_abort == 0;
      if (EIGHT) {
        mls[w][row] = kept_ml;
        if (w == 0) descs[row] = RowDesc{kept.off, kept_t, kept.anc};
      }
      if (!has) mls[w][row] = make_float2(-INFINITY, 0.f);
      if (has && 32 * (warp & 3) < rows_blk) {
        const uint32_t tl = tmem + (uint32_t(32 * (warp & 3)) << 16) + 256u * w;
#pragma unroll 1
        for (int c = 0; c < D / 32; ++c) {
          uint32_t ov[32];
          tc::tmem_ld32(tl + C::O_COL + c * 32, ov);
          tc::tmem_wait_ld();
#pragma unroll
          for (int e = 0; e < 8; ++e)
            *reinterpret_cast<uint4 *>(part + (w * ROWS + row) * D + (((c * 8 + e) ^ (row & (CH - 1))) << 2)) =
                make_uint4(ov[4 * e], ov[4 * e + 1], ov[4 * e + 2], ov[4 * e + 3]);
        }
      }
    }
    tc::fence_before_sync();
    __syncwarp();
    if (nsplit > 1) cluster_sync();
    else __syncthreads();
    const int parts = 2 * nsplit;
    const uint32_t ml_a = smem_u32(mls), part_a = smem_u32(part), ab_a = smem_u32(&s_abort), dirty_a = smem_u32(&s_dirty[0]);
    // part i: slot i & 1 of CTA i >> 1
    int state = 0;  // 1: a CTA gave up, 2: done again row by row
    if (lane < nsplit) {
      uint32_t ab, di;
      asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(ab) : "r"(mapa(ab_a, lane)) : "memory");
      asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(di) : "r"(mapa(dirty_a, lane)) : "memory");
      state = (ab ? 1 : 0) | (di ? 2 : 0);
    }
    const bool gave_up = __any_sync(0xffffffffu, state & 1), again = __any_sync(0xffffffffu, state & 2);
    const bool first_has = m > 0;  // (a CTA without tiles has no row descriptions: it joins nothing)
    const int joiners = ::max(1, ::min(nsplit, it.n));
    if (!gave_up && first_has) {
      constexpr int WARPS = C::THREADS / 32, AHEAD = 8;
      auto sums = [&](int row) {
        return row < rows_blk && lane < parts ? ld_cluster2(mapa(ml_a + ((lane & 1) * ROWS + row) * 8, lane >> 1)) : make_float2(-INFINITY, 0.f);
      };
      float2 next = sums(split * WARPS + warp);
      for (int row = split * WARPS + warp; row < rows_blk; row += joiners * WARPS) {
        const float2 ml = next;
        next = sums(row + joiners * WARPS);
        const int off = descs[row].off, t = descs[row].t;
        if (off < 0) continue;  // a malformed tree
        const int h = it.g * p.G + row - (t - it.t00) * p.G;
        if (again || __any_sync(0xffffffffu, ml.y > MOST_SUM)) {
          slow_row<D, EIGHT>(P, it.b, it.g, it.L, t, h, off, descs[row].anc, &s_beat);
          continue;
        }
        const uint32_t some = __ballot_sync(0xffffffffu, ml.y != 0.f);
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f), v[AHEAD];
        auto fetch = [&](int i0) {  // parts of other CTAs take a while: many at once
#pragma unroll
          for (int k = 0; k < AHEAD; ++k) {
            const int i = i0 + k;
            v[k] = ((some >> i) & 1u) && lane < CH
                       ? ld_cluster4(mapa(part_a + (((i & 1) * ROWS + row) * D + ((lane ^ (row & (CH - 1))) << 2)) * 4, i >> 1))
                       : make_float4(0.f, 0.f, 0.f, 0.f);
          }
        };
        fetch(0);
        float M = ml.x;
#pragma unroll
        for (int k = 16; k > 0; k >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, k));
        const float c = ml.y == 0.f ? 0.f : tc::ex2(ml.x - M);
        float Z = ml.y == 0.f ? 0.f : c * ml.y;
#pragma unroll
        for (int k = 16; k > 0; k >>= 1) Z += __shfl_xor_sync(0xffffffffu, Z, k);
        for (int i0 = 0; i0 < parts; i0 += AHEAD) {
          if (i0 > 0) fetch(i0);
#pragma unroll
          for (int k = 0; k < AHEAD; ++k) {
            const float ci = __shfl_sync(0xffffffffu, c, i0 + k);
            acc.x += ci * v[k].x;
            acc.y += ci * v[k].y;
            acc.z += ci * v[k].z;
            acc.w += ci * v[k].w;
          }
        }
        if (__builtin_expect(__any_sync(0xffffffffu, ml.y > SAFE_SUM), 0)) {
          // (a sum of 0 x O is zero, or NaN)
          const float odd = 0.f * acc.x + 0.f * acc.y + 0.f * acc.z + 0.f * acc.w;
          if (__any_sync(0xffffffffu, odd != 0.f)) {  // (also where it is NaN)
            slow_row<D, EIGHT>(P, it.b, it.g, it.L, t, h, off, descs[row].anc, &s_beat);
            continue;
          }
        }
        const float inv = 1.f / Z;
        const int64_t orow = (int64_t(it.b) * p.T_max + t) * p.Hq + h;
        if (lane < CH)
          *reinterpret_cast<uint2 *>(p.out + orow * D + lane * 4) =
              make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
        if (lane == 0 && p.lse != nullptr) p.lse[orow] = (M + log2f(Z)) * LN2;
      }
    }
    __syncwarp();
    if (nsplit > 1) cluster_sync();  // no CTA leaves while another reads its shared memory
    else __syncthreads();
    tc::fence_after_sync();
  }
  if (warp == MMA_WARP) {
    __syncwarp();
    tc::tmem_dealloc(tmem, TMEM_COLS);
  }
}

// ------------------------------------------------------------------ host side
// (64 columns, 1 head, 64 slots, 1) boxes of one layer's K or V, 128-byte swizzle;
// boxes outside read as zeros. Contiguous: (D, Hkv, capacity, B); paged: (D, Hkv,
// 64, num_pages).
bool kv_map(CUtensorMap *m, const void *base, const WinParams &p, int D) {
  EncodeTiledFn enc = encode_tiled();
  if (enc == nullptr) return false;
  const bool paged = p.table != nullptr;
  const cuuint64_t slots = paged ? 64 : cuuint64_t(p.capacity), outer = paged ? cuuint64_t(p.num_pages) : cuuint64_t(p.B);
  const cuuint64_t dims[4] = {cuuint64_t(D), cuuint64_t(p.Hkv), slots, outer};
  const cuuint64_t strides[3] = {cuuint64_t(D) * 2, cuuint64_t(p.Hkv) * D * 2, slots * p.Hkv * D * 2};
  const cuuint32_t box[4] = {64, 1, 64, 1}, one[4] = {1, 1, 1, 1};
  return enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void *>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The rows of a block, (token, head) in order: (64 columns, G heads, 1 KV head, TB
// tokens, 1) boxes of (D, G, Hkv, T_max, B).
bool q_map(CUtensorMap *m, const WinParams &p, int D, int TB) {
  EncodeTiledFn enc = encode_tiled();
  if (enc == nullptr) return false;
  const cuuint64_t dims[5] = {cuuint64_t(D), cuuint64_t(p.G), cuuint64_t(p.Hkv), cuuint64_t(p.T_max), cuuint64_t(p.B)};
  const cuuint64_t strides[4] = {cuuint64_t(D) * 2, cuuint64_t(p.G) * D * 2, cuuint64_t(p.st) * 2, cuuint64_t(p.sb) * 2};
  const cuuint32_t box[5] = {64, cuuint32_t(p.G), 1, cuuint32_t(TB), 1}, one[5] = {1, 1, 1, 1, 1};
  return enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<__nv_bfloat16 *>(p.q), dims, strides, box, one,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Codes of one layer's K or V: (D, 1 head, 64 slots, 1) boxes of (D, Hkv, 64, num_pages),
// rows one behind the other.
bool code_map(CUtensorMap *m, const uint8_t *base, const WinParams &p, const Kv8 &c, int D) {
  EncodeTiledFn enc = encode_tiled();
  if (enc == nullptr) return false;
  const cuuint64_t dims[4] = {cuuint64_t(D), cuuint64_t(p.Hkv), 64, cuuint64_t(c.num_pages)};
  const cuuint64_t strides[3] = {cuuint64_t(D), cuuint64_t(p.Hkv) * D, cuuint64_t(64) * p.Hkv * D};
  const cuuint32_t box[4] = {cuuint32_t(D), 1, 64, 1}, one[4] = {1, 1, 1, 1};
  return enc(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, const_cast<uint8_t *>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, bool PAIR, bool EIGHT, bool CLUSTER = false>
dreams_status_t launch(ParamsOf<EIGHT> &P, cudaStream_t stream) {
  using C = Cfg<D, PAIR, EIGHT>;
  const void *kernel = reinterpret_cast<const void *>(window_tc_kernel<D, PAIR, EIGHT, CLUSTER>);
  const dreams_status_t st = ensure_max_dynamic_smem(kernel, int(C::SMEM));
  if (st != DREAMS_OK) return st;
  if (!kv_map(&P.tmap_k, P.p.k, P.p, D) || !kv_map(&P.tmap_v, P.p.v, P.p, D) || !q_map(&P.tmap_q, P.p, D, P.TB)) return DREAMS_ERR_UNSUPPORTED;
  if constexpr (EIGHT) {
    if (!code_map(&P.tmap_k8, P.c.k, P.p, P.c, D) || !code_map(&P.tmap_v8, P.c.v, P.p, P.c, D)) return DREAMS_ERR_UNSUPPORTED;
  }
  cudaLaunchConfig_t cfg = {};
  if constexpr (CLUSTER) cfg.gridDim = dim3(2u * unsigned(std::min(P.items, P.clusters)));
  else cfg.gridDim = dim3(PAIR ? unsigned(std::min(P.items, num_sms())) : unsigned(P.items) * unsigned(P.p.nsplit));
  cfg.blockDim = dim3(C::THREADS);
  cfg.dynamicSmemBytes = C::SMEM;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2] = {early_launch()};
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = unsigned(P.p.nsplit);
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = P.p.nsplit > 1 ? 2 : 1;
  void *args[] = {&P};
  const cudaError_t e = cudaLaunchKernelExC(&cfg, kernel, args);
  if (e != cudaSuccess) {
    set_last_cuda_error(e);
    return DREAMS_ERR_CUDA;
  }
  return check_launch();
}

// How many clusters of ns CTAs the current device runs at once (asked once per
// device); 0: none, or not known.
template <int D, bool EIGHT, bool PAIR = false>
int clusters_at_once(int ns) {
  using C = Cfg<D, PAIR, EIGHT>;
  static std::atomic<int> known[64][9];  // count + 1
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev >= 64) return 0;
  int n = known[dev][ns].load(std::memory_order_relaxed);
  if (n == 0) {
    const void *kernel = reinterpret_cast<const void *>(window_tc_kernel<D, PAIR, EIGHT, PAIR>);
    if (ensure_max_dynamic_smem(kernel, int(C::SMEM)) != DREAMS_OK) return 0;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(ns));
    cfg.blockDim = dim3(C::THREADS);
    cfg.dynamicSmemBytes = C::SMEM;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = unsigned(ns);
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess) {
      cudaGetLastError();
      n = 0;
    }
    known[dev][ns].store(++n, std::memory_order_relaxed);
  }
  return n - 1;
}

template <bool EIGHT>
dreams_status_t launch_blocks(ParamsOf<EIGHT> &P, int D, cudaStream_t stream) {
  const WinParams &p = P.p;
  P.TB = std::max(1, ROWS / p.G);
  const int64_t heads = int64_t(p.B) * p.Hkv;
  const int64_t blocks = (int64_t(p.T_max) + P.TB - 1) / P.TB, pairs = (blocks + 1) / 2;
  test_stall(DREAMS_TEST_ATTENTION, &P.stall_at, &P.wait_ns);
  // Columns of a block (its keys begin anywhere in a page), and the time of either
  // layout in tenths of a microsecond, from sweeps of both over 5 to 33 tiles and 8 to
  // 448 blocks: a CTA of a block takes 13.5 us and 1.5 (head dim 64: 1.3) a tile, a
  // round of them after the other; a pair of blocks 2 (1.6) a tile, 3 to change items
  // and 4 once. 17 tiles: trees of 16 sequences, 128 pairs 45 us, 256 blocks 85; 9
  // tiles: a tree's 32 blocks 22 us, over clusters of 4 13.5.
  // A later sweep of both (32 to 864 blocks, windows of 512 to 4096) has pairs as said (1.4
  // a tile with head dim 64), a CTA of a block at 12.6 and 1.5 (64: 15.4 and 0.85), and
  // one of a cluster of 4 at 10 and 1.2: the rule overrates clusters by 3 to 6 us. It took
  // the slower layout at 5 of 96 points, all near where the two cross: 18.3 us against
  // 15.7 (64 blocks, 5 tiles), 14.6 against 11.8 (32 blocks, 5 tiles, head dim 64), and 4
  // to 7% at 17 tiles of 96 to 152 blocks with head dim 64.
  const int64_t sms = num_sms();
  const int64_t keys = std::min<int64_t>(p.capacity, int64_t(p.window) + std::min<int64_t>(p.T_max, P.TB));
  const int64_t cols = keys + 63 + (std::min<int64_t>(p.capacity, p.sinks) + 63) / 64 * 64 + 32;
  const int64_t per_one = D == 128 ? 15 : 13, per_pair = D == 128 ? 20 : 16;
  auto rounds = [](int64_t n, int64_t fit) { return (n + fit - 1) / fit; };
  const int64_t pair_cost = blocks > 1 ? rounds(heads * pairs, sms) * (per_pair * cols / KT + 30) + 40 : INT64_MAX;
  int64_t best = INT64_MAX;
  int nsplit = 1;
  for (int ns = 1; ns <= 8 && (ns == 1 || (ns * KT <= cols && heads * blocks * ns <= sms)); ++ns) {
    const int64_t fit = ns == 1 ? sms : D == 128 ? clusters_at_once<128, EIGHT>(ns) : clusters_at_once<64, EIGHT>(ns);
    if (fit < 1) continue;
    const int64_t cost = rounds(heads * blocks, fit) * (135 + per_one * (cols + (ns - 1) * KT / 2) / (ns * KT));
    if (cost < best) {
      best = cost;
      nsplit = ns;
    }
  }
  bool pair = pair_cost <= best, cluster = false;
  if constexpr (EIGHT) {
    // Pairs of blocks on clusters of two CTAs. Up to a pair for each cluster that runs at
    // once, each is cut in half: 12.5 us and 2.45 a tile of a CTA (head dim 64: 11.5 and 1.95).
    // Above, where at least one SM in eight would have nothing to do and the lengths may
    // differ, the halves of the longest have the shortest beside them. Against pairs or
    // blocks as above, trees of 64 nodes, 8 KV heads, head dim 128, us:
    //   pairs                  32          64         96         128        152
    //   of 1500 to 6000   57.5 59.8  117.2 68.1  112.5 74.7  113.0 93.3  117.1 107.3
    //   of 4000           44.8 47.9   85.4 52.2   80.7 86.4   80.9 88.5   88.1  93.5
    //   of 2000 to 3000   34.3 38.6   65.5 42.2   61.9 56.3   62.4 69.6   65.7  75.6
    // (At 128 and 152 all SMs run, and a tile takes 2.35 us where it takes 2.15 with 128.)
    P.clusters = D == 128 ? clusters_at_once<128, true, true>(2) : clusters_at_once<64, true, true>(2);
    const int64_t n = heads * pairs;
    if (blocks > 1 && n <= P.clusters) cluster = 10 * (D == 128 ? 125 : 115) + (D == 128 ? 245 : 195) * cols / (2 * KT) < 10 * std::min(best, pair_cost);
    else cluster = pair && p.B > 1 && n <= std::min<int64_t>(2 * P.clusters, sms - sms / 8);
  }
  pair = pair || cluster;
  P.p.nsplit = cluster ? 2 : pair ? 1 : nsplit;
  P.nblk = int(pair ? pairs : blocks);
  const int64_t items = heads * P.nblk;
  if (items * P.p.nsplit > INT_MAX / 2) return DREAMS_ERR_UNSUPPORTED;
  P.items = int(items);
  P.heads = Divisor::of(heads);
  P.hkv = Divisor::of(p.Hkv);
  P.nsplit = Divisor::of(P.p.nsplit);
  P.g = Divisor::of(p.G);
  if constexpr (EIGHT) {
    P.seqs = Divisor::of(p.B);
    P.ranked = cluster || (pair && items > sms && int64_t(P.nblk) * p.B <= MAX_RANKED);
    if (cluster) return D == 128 ? launch<128, true, true, true>(P, stream) : launch<64, true, true, true>(P, stream);
  }
  if (D == 128) return pair ? launch<128, true, EIGHT>(P, stream) : launch<128, false, EIGHT>(P, stream);
  return pair ? launch<64, true, EIGHT>(P, stream) : launch<64, false, EIGHT>(P, stream);
}

}  // namespace

dreams_status_t launch_tc(const WinParams &p, const dreams_kv_cache_t *kv, cudaStream_t stream) {
  TcParams P;
  memset(&P, 0, sizeof(P));
  P.p = p;
  return launch_blocks<false>(P, kv->D, stream);
}

dreams_status_t launch_tc8(const WinParams &p, const Kv8 &c, int D, cudaStream_t stream) {
  Tc8Params P;
  memset(&P, 0, sizeof(P));
  P.p = p;
  P.c = c;
  return launch_blocks<true>(P, D, stream);
}

}  // namespace win
}  // namespace dreams
