// Attention of a few query rows over a paged cache (single tokens, short
// chunks), and the join of keys that were split over blocks.
//
// HBM-bound: each cached K and V row is read once per row tile, 8 or 16 query
// rows (the query heads that share a KV head, times the new tokens) use it.
// Blocks of 4 warps, as many as fit the device, take equal shares of all steps of
// 32 keys. Each warp takes steps of its own: it copies them into its own ring of
// shared-memory stages (cp.async, no block barrier anywhere in the loop) and
// keeps its own softmax state; the warps join at the end of a row tile's keys, and
// a second kernel joins the parts where several blocks share a tile.
//
// Keys are the matrix instructions' long side, S^T = K Q^T and O^T = V^T P^T
// (mma.m16n8k16 with 16 keys or channels by 8 query rows), so 7 or 8 query
// rows fill a tile that row-major scores would leave half empty. A thread's
// accumulators of S^T and O^T belong to the same two query rows, so the running
// maximum rescales in place, and S^T becomes the second product's operand by
// one 8x8 transpose (movmatrix).
//
// Codes go into the fp16 matrix instruction as they are: a code u masked into a
// 16-bit lane is the subnormal fp16 u * 2^-24 (or 16u * 2^-24), exact. The
// K side's steps and minima are applied to the sums: q . k = sum over groups
// of s_g (q_g . u_g) + m_g sum(q_g). Query rows are scaled by a power of two
// into fp16's range. On the V side the steps go into the weights, one operand
// for each group: out = sum_j (p_j s_gj) u_j + sum_j p_j m_gj, the second sum a
// number per query row and group. The products p s are rounded to fp16 (11 bits)
// after a power of two that keeps the largest step's below 2^15. So a code costs
// a mask and its share of two byte permutations and a shift, no multiplication.
//
// Measured: one token for each of 8 streams, 24576 bf16 rows, 8 KV heads of 8 query
// heads: 124 us, 6.5 TB/s (96% of the copy bandwidth); 32 streams of up to 24577
// 4-bit rows: 124 us, 4.3 TB/s: no unit is busy more than 56% (issue; DRAM 51%, ALU 50%:
// masks, permutations, addresses), 12 warps per SM wait in a step's chain; 32 streams of 12288 8-bit rows: 148 us, 5.8 TB/s.
#pragma once

#include <cuda_fp16.h>

#include "attend_share.cuh"
#include "paged.cuh"

namespace ipv {
namespace {

constexpr int kThreads = 32 * kRowsWarps;
constexpr int kRunCost = 6;  // what a run of steps costs beside them, in steps
constexpr int kCluster = kRowsCluster;
constexpr float kNegInf = -INFINITY;

template <int FMT, int DP>
struct Ring {
  static constexpr int kRowB = FMT == kBf16 ? DP * 2 : FMT == kU8 ? DP : DP / 2;  // bytes of a row
  static constexpr int kTile = kRowsStep * kRowB;
  static constexpr int kG = DP / kGroup;
  static constexpr int kPar = FMT == kBf16 ? 0 : kRowsStep * kG * 4;
  static constexpr int kStage = 2 * kTile + 2 * kPar;
  // bf16: 96 to 128 KB in flight with one block per SM; codes: 3 blocks, and 3 stages
  // were slower (32 streams of 12288 8-bit rows 213 us against 150).
  static constexpr int kStages = FMT == kBf16 ? 3 : 2;
};

// How a kernel lays itself out. Over all pages, blocks per SM: bf16 at 128 channels has enough bytes in flight with one, codes
// need warps to widen them (32 ragged 4-bit streams: 3 blocks of 168 registers 123 us, 4 of 128, with spills, 134). Chosen pages of 128 channels are mostly found in L2, and a tile has few steps: what counts is
// how many warps there are, and that other blocks go on while one starts a tile or joins its warps. bf16: rings of two halves of
// a stage, K's and V's, each refilled as soon as it has been read, the warps' results in their place at a tile's end, and three
// blocks per SM (questions of 8 streams 66 us; two blocks with 3 halves and the next tile on its way 84, one of 8 warps 103, of
// 4 with 3 stages 126). 8-bit codes: 3 halves and the results behind them, three blocks per SM instead of two (200 streams'
// tokens 154 us against 169, questions 96 against 105; 32 streams', a block each, 35 against 32). Three blocks leave 168
// registers, of which the chosen instances for 8 query rows over 8 and 4 bits at 128 channels want a few more (92 and 48 bytes spilled).
template <int FMT, int DP, int NR, bool CHOSEN>
struct Layout {
  static constexpr bool kHalves = CHOSEN && FMT != kU4 && DP == 128 && NR == 1;
  static constexpr bool kTwo = kHalves && FMT == kBf16;  // halves; results in their place
  static constexpr int kBlocks = kHalves ? 3 : FMT == kBf16 && DP == 128 ? 1 : NR == 1 ? 3 : 2;  // per SM
  static constexpr int kHalf = Ring<FMT, DP>::kTile + (FMT == kBf16 ? 0 : Ring<FMT, DP>::kPar);  // K's or V's rows, their pairs
  static constexpr int kRing = kHalves ? (kTwo ? 2 : 3) * kHalf : Ring<FMT, DP>::kStage * Ring<FMT, DP>::kStages;  // of a warp
  static constexpr int kRings = kRing * kRowsWarps;
  // The warps' results: [rows][kPitch] sums each, maxima and sums of weights; a cluster's part.
  static constexpr int kPitch = DP + 4, kResult = 8 * NR * kPitch * 4;
  static constexpr int kResults = kTwo ? 0 : kRings, kResultApart = kTwo ? kRing : kResult;
  static constexpr int kStats = kTwo ? kRings : kRings + kRowsWarps * kResult;
  static constexpr int kPart = kTwo ? kHalf : 0;
  static constexpr int kBytes = kStats + kRowsWarps * 8 * NR * 2 * 4;
  static_assert(!kTwo || kResult <= kHalf, "a warp's results take the first of its halves, the part the other");
};

// Where 16-byte chunk c of key row r lies in its row: the rows that a quarter
// or half warp reads at once come to lie in different banks.
template <int FMT, int RB>
__device__ __forceinline__ int swizzle(int r, int c) {
  if (FMT == kBf16) return c ^ (r & 7);
  if (RB == 128) return c ^ (2 * (r & 3)) ^ (r & 4);
  if (RB == 64) return c ^ ((((r >> 1) ^ (r >> 2)) & 1) << 1);
  return c;
}

// Key of the 16 of a tile that stands at matrix row i. With codes, rows 2t and
// 2t + 1 are keys t and t + 4, which keeps a half warp's V rows in different
// banks; with bf16 ldmatrix wants no such thing.
template <int FMT>
__device__ __forceinline__ int key_at(int i) {
  if (FMT == kBf16) return i;
  return (i & 8) | ((i & 7) >> 1) | ((i & 1) << 2);
}

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool ok) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(ok ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy16_at(uint32_t dst, const char* src, int offset) {  // a constant offset
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src + offset) : "memory");
}
template <int N>
__device__ __forceinline__ void copy_small(uint32_t dst, const void* src, bool ok) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(N), "r"(ok ? N : 0) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(at)
               : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(at)
               : "memory");
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
template <bool BF16>
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if (BF16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
template <bool BF16>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  uint32_t r;
  if (BF16)
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  else
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t lds32(uint32_t at) {
  uint32_t v;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t at) {
  uint2 v;
  asm volatile("ld.shared.v2.b32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ uint4 lds128(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ __half2 as_half2(uint32_t x) { return *reinterpret_cast<__half2*>(&x); }
__device__ __forceinline__ float par_step(uint32_t p) { return __low2float(as_half2(p)); }
__device__ __forceinline__ float par_min(uint32_t p) { return __high2float(as_half2(p)); }

// Channel of accumulator row (tile ct, half) of the thread in lane group g of
// the second product: with codes, the channels whose codes the thread reads,
// four tiles for each group of channels.
template <int FMT>
__device__ __forceinline__ int out_channel(int ct, int half, int g) {
  if (FMT == kBf16) return ct * 16 + half * 8 + g;
  const int gr = (ct >> 2) * kGroup, t = g >> 1;
  if (FMT == kU8) return gr + 4 * (t + 4 * (2 * (g & 1) + ((ct >> 1) & 1))) + 2 * (ct & 1) + half;
  return gr + 8 * (t + 4 * (g & 1)) + 2 * (ct & 3) + half;
}

// Four channels, from c on, of query row r of a sequence's KV head.
__device__ __forceinline__ void write_row(const AttendArgs& a, const Seq& s, int head, int r, int c, const float4& acc, float top,
                                          float sum) {
  const int tok = a.by_share(r), hq = head * a.share + r - tok * a.share;
  const int64_t row = s.row0 + static_cast<int64_t>(tok);
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  if (c < a.p.dim)
    *reinterpret_cast<uint2*>(a.out + row * a.out_row + hq * a.out_head + c) =
        make_uint2(pack2<true>(acc.x * inv, acc.y * inv), pack2<true>(acc.z * inv, acc.w * inv));
  if (c == 0 && a.lse) a.lse[row * a.q_heads + hq] = sum == 0.0f ? kNegInf : (top + log2f(sum)) * 0.6931471805599453f;
}

// Clusters: a block's rank, the address of a shared-memory word in block r of
// the cluster, loads from there, and the barrier of all blocks.
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t in_block(uint32_t at, uint32_t r) {
  uint32_t x;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(x) : "r"(at), "r"(r));
  return x;
}
__device__ __forceinline__ float4 far128(uint32_t at) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ float2 far64(uint32_t at) {
  float2 v;
  asm volatile("ld.shared::cluster.v2.f32 {%0,%1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// CHOSEN: a row tile's keys are those of its new row's chosen pages, one list for each KV head.
template <int FMT, int DP, int NR, bool CHOSEN>
__global__ void __launch_bounds__(kThreads, (Layout<FMT, DP, NR, CHOSEN>::kBlocks)) attend_rows_kernel(AttendArgs a, int tiles) {
  using R = Ring<FMT, DP>;
  using L = Layout<FMT, DP, NR, CHOSEN>;
  constexpr int kWarps = kRowsWarps;
  constexpr bool kB = FMT == kBf16;
  constexpr int kCh = R::kRowB / 16;     // chunks of a row
  constexpr int kKs = DP / 16;           // k-steps of the first product
  constexpr int kCt = DP / 16;           // channel tiles of the second
  constexpr int kG = kB ? 1 : R::kG;     // accumulators of the first product
  extern __shared__ __align__(128) unsigned char smem[];

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  constexpr int kTileRows = 8 * NR;
  pdl_wait();
  const Share share = find_share<kTileRows, kRowsStep, kRunCost, kThreads, CHOSEN>(a, tiles, reinterpret_cast<int64_t*>(smem));
  int slots = 0;  // partial results used
  const bool clustered = a.unit == 0 && a.cluster > 1;
  if (share.left <= 0 && !clustered) {
    if (threadIdx.x < 2 && a.unit > 0) a.part_rec[2 * blockIdx.x + threadIdx.x] = make_int4(0, 0, 0, 0);
    return;
  }
  __syncthreads();  // the shared memory held find_share's scratch
  using W = Walk<kTileRows, kRowsStep, kRunCost, CHOSEN>;
  W w = {};
  const uint32_t ring = smem_u32(smem) + warp * L::kRing;
  const int nch = a.p.row_bytes >> 4;

  // ---- copies of one step into one stage (this warp's lanes only)
  // A lane's chunks are chunk my_c of keys my_r, my_r + 32 / kCh, ...
  constexpr int kApart = 32 / kCh;
  const int my_r = lane / kCh, my_c = lane % kCh;
  const int64_t v_from_k = a.p.v - a.p.k;
  const int64_t page_bytes = a.p.page_stride * a.p.row_bytes, next_bytes = a.p.row_stride * a.p.row_bytes;
  // This lane's key of step i of run x: its page, -1: none. Read a step ahead of the copies.
  auto page_of = [&](const W& x, int i) {
    const int j = x.t.kr.template key0<kRowsStep>(i) + lane;
    int pg = -1;
    if (i < x.s + x.n && j < x.t.kr.hi_max) pg = a.p.table ? a.p.table[x.t.b * a.p.table_stride + (j >> a.p.page_shift)] : x.t.b;
    return static_cast<unsigned>(pg) < static_cast<unsigned>(a.p.n_pages) ? pg : -1;
  };
  auto issue = [&](const W& x, int i, int pg, int stage) {
    const uint32_t base = ring + stage * R::kStage;
    const int j = x.t.kr.template key0<kRowsStep>(i) + lane;
    const int64_t head_rows = x.head * a.p.head_stride;
    const int64_t off = pg < 0 ? int64_t{-1}
                               : head_rows * a.p.row_bytes + pg * page_bytes +
                                     (a.p.page_shift == 31 ? j : j & (a.p.page_size - 1)) * next_bytes;
    if constexpr (!kB) {
      constexpr int kN = R::kG * 4;
      const int64_t at = pg < 0 ? 0 : off / (R::kRowB / kN);  // a row of codes is 8 or 16 times its pairs
      copy_small<kN>(base + 2 * R::kTile + lane * kN, reinterpret_cast<const char*>(a.p.k_par) + at, pg >= 0);
      copy_small<kN>(base + 2 * R::kTile + R::kPar + lane * kN, reinterpret_cast<const char*>(a.p.v_par) + at, pg >= 0);
    }
#pragma unroll
    for (int u = 0; u < kCh; ++u) {
      const int r = u * kApart + my_r;
      const int64_t at = __shfl_sync(0xffffffffu, off, r);
      const bool ok = at >= 0 && (!kB || my_c < nch);
      const char* src = ok ? a.p.k + my_c * 16 + at : a.p.k;
      const uint32_t dst = base + r * R::kRowB + swizzle<FMT, R::kRowB>(r, my_c) * 16;
      copy16(dst, src, ok);
      copy16(dst + R::kTile, src + v_from_k, ok);
    }
  };
  // Chosen pages: 16 keys of a step lie in one page. Lane l looks up the page (-1: none of the pool, its rows read as zero),
  // and how many of its keys are seen, of keys (l & 16).. of this warp's step k0 + (l & 15): two dependent loads
  // for 16 steps, no 64-bit products and few shuffles for each.
  int page_l = -1, seen_l = 0;
  auto look_up = [&](const W& x, int k0) {
    const int i = x.s + warp + (k0 + (lane & 15)) * kWarps, j = x.t.kr.template key0<kRowsStep>(i) + (lane & 16);
    page_l = -1, seen_l = 0;
    if (i < x.s + x.n && j < x.t.kr.hi_max) {
      const int tok = a.by_share(x.t.row0), hi = token_hi(a, x.t.seq, tok);
      const int c = a.chosen[(x.t.seq.row0 + static_cast<int64_t>(tok)) * a.chosen_row + x.head * a.chosen_head + (j >> a.p.page_shift)];
      if (static_cast<unsigned>(c) < static_cast<unsigned>(pages_seen(a, x.t.seq, tok))) {
        const int pg = a.p.table ? a.p.table[x.t.b * a.p.table_stride + c] : x.t.b;
        if (static_cast<unsigned>(pg) < static_cast<unsigned>(a.p.n_pages)) page_l = pg;
        seen_l = a.p.page_shift == 31 ? hi : min(hi - (c << a.p.page_shift), a.p.page_size);
      }
    }
  };
  // Where the two halves of this warp's step k lie, how many of their 16 rows are to be copied, which keys are seen.
  struct Halves {
    int64_t at[2];
    int n[2];
    uint32_t seen;
  };
  auto halves = [&](const W& x, int k) {
    Halves h;
    h.seen = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int pg = __shfl_sync(0xffffffffu, page_l, (k & 15) + 16 * i), upto = __shfl_sync(0xffffffffu, seen_l, (k & 15) + 16 * i);
      const int j = x.t.kr.template key0<kRowsStep>(x.s + warp + k * kWarps) + 16 * i;
      const int in = a.p.page_shift == 31 ? j : j & (a.p.page_size - 1), n = min(max(upto - in, 0), 16);
      h.n[i] = pg < 0 ? 0 : n;
      h.at[i] = x.head * a.p.head_stride * a.p.row_bytes + pg * page_bytes + in * next_bytes;
      h.seen |= ((1u << n) - 1u) << (16 * i);
    }
    return h;
  };
  const int64_t lane_at = my_r * next_bytes + my_c * 16;
  const int lane_row = my_c < nch ? my_r : 16;  // 16: never copied
  // Rows without gaps and all there, as most: offsets that are known here, one instruction or two for each copy.
  const bool dense = next_bytes == R::kRowB && a.p.row_bytes == R::kRowB;
  auto copy_rows = [&](const char* from, uint32_t to, const Halves& h) {
    if (dense && min(h.n[0], h.n[1]) == 16) {
      const char* src[2] = {from + h.at[0] + lane_at, from + h.at[1] + lane_at};
#pragma unroll
      for (int u = 0; u < kCh; ++u)
        copy16_at(to + (u * kApart + my_r) * R::kRowB + swizzle<FMT, R::kRowB>(u * kApart + my_r, my_c) * 16, src[u * kApart / 16],
                  u * kApart % 16 * R::kRowB);
      return;
    }
#pragma unroll 1
    for (int u = 0; u < kCh; ++u) {
      const bool up = u * kApart >= 16;
      const int r = u * kApart - (up ? 16 : 0);
      const bool ok = lane_row + r < (up ? h.n[1] : h.n[0]);
      copy16(to + (u * kApart + my_r) * R::kRowB + swizzle<FMT, R::kRowB>(u * kApart + my_r, my_c) * 16,
             ok ? from + ((up ? h.at[1] : h.at[0]) + r * next_bytes + lane_at) : from, ok);
    }
  };
  // Codes: the pairs of this lane's row, in bytes from a pool's first; -1: not to be copied.
  constexpr int kPairB = kB ? 4 : R::kG * 4;
  auto pairs_at = [&](const Halves& h) {
    const bool ok = (lane & 15) < (lane < 16 ? h.n[0] : h.n[1]);
    return ok ? ((lane < 16 ? h.at[0] : h.at[1]) + (lane & 15) * next_bytes) / (R::kRowB / kPairB) : int64_t{-1};
  };
  auto copy_pairs = [&](const uint32_t* par, uint32_t to, int64_t at) {
    copy_small<kPairB>(to + lane * kPairB, reinterpret_cast<const char*>(par) + max(at, int64_t{0}), at >= 0);
  };
  auto issue_chosen = [&](const Halves& h, int stage) {
    const uint32_t base = ring + stage * R::kStage;
    if constexpr (!kB) {
      const int64_t at = pairs_at(h);
      copy_pairs(a.p.k_par, base + 2 * R::kTile, at);
      copy_pairs(a.p.v_par, base + 2 * R::kTile + R::kPar, at);
    }
    copy_rows(a.p.k, base, h);
    copy_rows(a.p.v, base + R::kTile, h);
  };
  auto copy_half = [&](const char* from, const uint32_t* par, int half, const Halves& h) {
    if constexpr (!kB) copy_pairs(par, ring + half * L::kHalf + R::kTile, pairs_at(h));
    copy_rows(from, ring + half * L::kHalf, h);
  };
  auto copy_k = [&](int half, const Halves& h) { copy_half(a.p.k, a.p.k_par, half, h); };
  auto copy_v = [&](int half, const Halves& h) { copy_half(a.p.v, a.p.v_par, half, h); };
  uint32_t seen_now = 0, seen_next = 0, seen_last = 0;  // keys of the step at hand and of the ones after it
  // The first steps of a run, and the page of the one after them.
  int page_next = -1;
  auto fill = [&](const W& x) {
    if constexpr (CHOSEN) {
      look_up(x, 0);
      const int end = x.n - warp;  // steps of the run from this warp's first on
      const Halves h0 = halves(x, 0);
      seen_now = h0.seen;
      if constexpr (L::kTwo) {
        if (end > 0) copy_k(0, h0);
        copy_commit();
        if (end > 0) copy_v(1, h0);
        copy_commit();
      } else if constexpr (L::kHalves) {  // K and V of the first step, K of the second
        const Halves h1 = halves(x, 1);
        seen_next = h1.seen;
        if (end > 0) copy_k(0, h0);
        copy_commit();
        if (end > 0) copy_v(1, h0);
        copy_commit();
        if (end > kWarps) copy_k(2, h1);
        copy_commit();
      } else {
#pragma unroll
        for (int i = 0; i < R::kStages - 1; ++i) {
          const Halves h = i == 0 ? h0 : halves(x, i);
          if (i == 1) seen_next = h.seen;
          if (end > i * kWarps) issue_chosen(h, i);
          copy_commit();
        }
      }
    } else {
      int pages[R::kStages];  // all on their way at once
#pragma unroll
      for (int i = 0; i < R::kStages; ++i) pages[i] = page_of(x, x.s + warp + i * kWarps);
#pragma unroll
      for (int i = 0; i < R::kStages - 1; ++i) {
        const int step = x.s + warp + i * kWarps;
        if (step < x.s + x.n) issue(x, step, pages[i], i);
        copy_commit();
      }
      page_next = pages[R::kStages - 1];
    }
  };

  // A cluster's part: [rows][DP sums, maximum, sum] in the rings, which one run leaves free.
  constexpr int kPartPitch = DP + 4;
  float* part_rows = reinterpret_cast<float*>(smem + L::kPart);

  bool go = share.left > 0 && w.begin(a, tiles, share);
  if (go) fill(w);
  for (int run = 0; go; ++run) {
    const Seq seq = w.t.seq;
    const KeyRange kr = w.t.kr;
    const int head = w.head;
    const int row0 = w.t.row0, row1 = row0 + w.t.n_rows - 1;
    const int first = w.s + warp, s_end = w.s + w.n;

    // ---- the query rows as the first product's second operand
    uint32_t qb[kKs][NR][2];
    float c_acc[NR][2], c_min[NR][2][kG];  // codes: factors of a thread's two rows
#pragma unroll
    for (int nr = 0; nr < NR; ++nr) {
      const int r = row0 + nr * 8 + g;
      const bool in = r <= row1;
      const int tok = a.by_share(in ? r : row0), hq = (in ? r : row0) - tok * a.share;
      const uint16_t* qp = a.q + (seq.row0 + static_cast<int64_t>(tok)) * a.q_row + (head * a.share + hq) * a.q_head;
      if constexpr (kB) {
#pragma unroll
        for (int ks = 0; ks < kKs; ++ks)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int ch = ks * 16 + i * 8 + 2 * t;
            qb[ks][nr][i] = in && ch < a.p.dim ? *reinterpret_cast<const uint32_t*>(qp + ch) : 0u;
          }
      } else {
        // The row's largest magnitude goes to [2^9, 2^10): its 1/16ths and its
        // products with subnormal codes keep all their bits. 4 threads share a row.
        uint32_t top = 0;
        for (int ch = 8 * t; ch < DP; ch += 32) {
          const uint4 x = in ? *reinterpret_cast<const uint4*>(qp + ch) : make_uint4(0, 0, 0, 0);
          const uint32_t xs[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
          for (int i = 0; i < 4; ++i) top = max(top, max(xs[i] & 0x7FFFu, (xs[i] >> 16) & 0x7FFFu));
        }
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const int e = min(max(static_cast<int>(top >> 7) - 127, -100), 126);
        const float up = __uint_as_float(static_cast<uint32_t>(127 + 9 - e) << 23);
        const float down = __uint_as_float(static_cast<uint32_t>(127 - 9 + e) << 23);
        auto load = [&](int ch, float f) {
          const float x = in ? __uint_as_float(static_cast<uint32_t>(qp[ch]) << 16) : 0.0f;
          return x * up * f;
        };
        float sum[kG];
#pragma unroll
        for (int gr = 0; gr < kG; ++gr) sum[gr] = 0.0f;
#pragma unroll
        for (int ks = 0; ks < kKs; ++ks) {
          const int gr = ks >> 2, w = FMT == kU8 ? ks & 3 : (ks >> 1) & 1;
          const bool hi4 = FMT == kU4 && (ks & 1);  // nibbles 1, 5, 3, 7 stand 4 bits up
          const float f = hi4 ? 0.0625f : 1.0f;
          const int c0 = gr * kGroup + (FMT == kU8 ? 4 : 8) * (t + 4 * w) + (hi4 ? 1 : 0);
          const int d = FMT == kU8 ? 2 : 4, d2 = FMT == kU8 ? 1 : 2;
          qb[ks][nr][0] = pack2<false>(load(c0, f), load(c0 + d, f));
          qb[ks][nr][1] = pack2<false>(load(c0 + d2, f), load(c0 + d2 + d, f));
          const __half2 s2a = as_half2(qb[ks][nr][0]), s2b = as_half2(qb[ks][nr][1]);
          sum[gr] += (__low2float(s2a) + __high2float(s2a) + __low2float(s2b) + __high2float(s2b)) * (hi4 ? 16.0f : 1.0f);
        }
        const float c = a.scale_log2 * down;
#pragma unroll
        for (int gr = 0; gr < kG; ++gr) {
          sum[gr] += __shfl_xor_sync(0xffffffffu, sum[gr], 1);
          sum[gr] += __shfl_xor_sync(0xffffffffu, sum[gr], 2);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          c_acc[nr][i] = __shfl_sync(0xffffffffu, c * 16777216.0f, 4 * (2 * t + i));
#pragma unroll
          for (int gr = 0; gr < kG; ++gr) c_min[nr][i][gr] = __shfl_sync(0xffffffffu, c * sum[gr], 4 * (2 * t + i));
        }
      }
    }

    // ---- what the thread's two rows of each row tile see
    int hi[NR][2];
#pragma unroll
    for (int nr = 0; nr < NR; ++nr)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = row0 + nr * 8 + 2 * t + i;
        hi[nr][i] = r <= row1 ? token_hi(a, seq, a.by_share(r)) : 0;
      }

    float o[kCt][NR][4];
    float m[NR][2], l[NR][2];
#pragma unroll
    for (int nr = 0; nr < NR; ++nr) {
      m[nr][0] = m[nr][1] = kNegInf;
      l[nr][0] = l[nr][1] = 0.0f;
#pragma unroll
      for (int ct = 0; ct < kCt; ++ct) o[ct][nr][0] = o[ct][nr][1] = o[ct][nr][2] = o[ct][nr][3] = 0.0f;
    }

    // Codes: sums of p m, and the largest step so far, as its fp16 exponent field;
    // weights times steps are held times 2^(29 - field).
    float pm[NR][2][kG];
#pragma unroll
    for (int nr = 0; nr < NR; ++nr)
#pragma unroll
      for (int gr = 0; gr < kG; ++gr) pm[nr][0][gr] = pm[nr][1][gr] = 0.0f;
    uint32_t field = 0;

    // ---- the loop over this warp's steps
    int stage = 0;
    int k_half = 0, v_half = 1, next_half = 2;  // halves: where K, V and the next step's K are
    int k = 0;                                  // chosen pages: which of this warp's steps it is
    for (int step = first; step < s_end; step += kWarps) {
      if constexpr (L::kHalves) {
        copy_wait<L::kTwo ? 1 : 2>();
      } else if constexpr (CHOSEN) {
        constexpr int kAhead = R::kStages - 1;
        if ((k + kAhead) % 16 == 0) look_up(w, k + kAhead);
        const Halves h = halves(w, k + kAhead);
        if (step + kAhead * kWarps < s_end) issue_chosen(h, stage == 0 ? kAhead : stage - 1);
        if (kAhead == 1) seen_next = h.seen; else seen_last = h.seen;
        copy_commit();
        copy_wait<kAhead>();
      } else {
        const int ahead = step + (R::kStages - 1) * kWarps;
        const int to = stage == 0 ? R::kStages - 1 : stage - 1;
        if (ahead < s_end) issue(w, ahead, page_next, to);
        page_next = page_of(w, ahead + kWarps);
        copy_commit();
        copy_wait<R::kStages - 1>();
      }
      __syncwarp();
      const uint32_t ks_at = ring + (L::kHalves ? k_half * L::kHalf : stage * R::kStage);
      const uint32_t vs_at = L::kHalves ? ring + v_half * L::kHalf : ks_at + R::kTile;
      const uint32_t kp_at = ks_at + (L::kHalves ? 1 : 2) * R::kTile, vp_at = L::kHalves ? vs_at + R::kTile : kp_at + R::kPar;
      const int key0 = kr.key0<kRowsStep>(step);

      float sc[2][NR][4];
      // S^T: 2 tiles of 16 keys
#pragma unroll
      for (int mt = 0; mt < 2; ++mt) {
        if constexpr (kB) {
#pragma unroll
          for (int nr = 0; nr < NR; ++nr) sc[mt][nr][0] = sc[mt][nr][1] = sc[mt][nr][2] = sc[mt][nr][3] = 0.0f;
          const int r = mt * 16 + (lane & 15);
#pragma unroll
          for (int ks = 0; ks < kKs; ++ks) {
            uint32_t ka[4];
            ldsm4(ka, ks_at + r * R::kRowB + swizzle<FMT, R::kRowB>(r, 2 * ks + (lane >> 4)) * 16);
#pragma unroll
            for (int nr = 0; nr < NR; ++nr) mma<true>(sc[mt][nr], ka, qb[ks][nr][0], qb[ks][nr][1]);
          }
#pragma unroll
          for (int nr = 0; nr < NR; ++nr)
#pragma unroll
            for (int i = 0; i < 4; ++i) sc[mt][nr][i] *= a.scale_log2;
        } else {
          float part[kG][NR][4];
#pragma unroll
          for (int gr = 0; gr < kG; ++gr)
#pragma unroll
            for (int nr = 0; nr < NR; ++nr) part[gr][nr][0] = part[gr][nr][1] = part[gr][nr][2] = part[gr][nr][3] = 0.0f;
          const int r0 = mt * 16 + key_at<FMT>(g), r1 = r0 + 8;
#pragma unroll
          for (int gr = 0; gr < kG; ++gr) {
            if constexpr (FMT == kU8) {
              const uint4 x = lds128(ks_at + r0 * R::kRowB + swizzle<FMT, R::kRowB>(r0, gr * 4 + t) * 16);
              const uint4 y = lds128(ks_at + r1 * R::kRowB + swizzle<FMT, R::kRowB>(r1, gr * 4 + t) * 16);
              const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
              for (int w = 0; w < 4; ++w) {
                const uint32_t ka[4] = {xs[w] & 0x00FF00FFu, ys[w] & 0x00FF00FFu, (xs[w] >> 8) & 0x00FF00FFu,
                                        (ys[w] >> 8) & 0x00FF00FFu};
#pragma unroll
                for (int nr = 0; nr < NR; ++nr) mma<false>(part[gr][nr], ka, qb[gr * 4 + w][nr][0], qb[gr * 4 + w][nr][1]);
              }
            } else {
              const int c = gr * 2 + (t >> 1), in = (t & 1) * 8;
              const uint2 x = lds64(ks_at + r0 * R::kRowB + swizzle<FMT, R::kRowB>(r0, c) * 16 + in);
              const uint2 y = lds64(ks_at + r1 * R::kRowB + swizzle<FMT, R::kRowB>(r1, c) * 16 + in);
              const uint32_t xs[2] = {x.x, x.y}, ys[2] = {y.x, y.y};
#pragma unroll
              for (int w = 0; w < 2; ++w) {
                const uint32_t xh = xs[w] >> 8, yh = ys[w] >> 8;
                const uint32_t k0[4] = {xs[w] & 0x000F000Fu, ys[w] & 0x000F000Fu, xh & 0x000F000Fu, yh & 0x000F000Fu};
                const uint32_t k1[4] = {xs[w] & 0x00F000F0u, ys[w] & 0x00F000F0u, xh & 0x00F000F0u, yh & 0x00F000F0u};
#pragma unroll
                for (int nr = 0; nr < NR; ++nr) {
                  mma<false>(part[gr][nr], k0, qb[gr * 4 + 2 * w][nr][0], qb[gr * 4 + 2 * w][nr][1]);
                  mma<false>(part[gr][nr], k1, qb[gr * 4 + 2 * w + 1][nr][0], qb[gr * 4 + 2 * w + 1][nr][1]);
                }
              }
            }
          }
          uint32_t p0[kG], p1[kG];
#pragma unroll
          for (int gr = 0; gr < kG; ++gr) {
            p0[gr] = lds32(kp_at + (r0 * kG + gr) * 4);
            p1[gr] = lds32(kp_at + (r1 * kG + gr) * 4);
          }
#pragma unroll
          for (int nr = 0; nr < NR; ++nr)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              float x = 0.0f, y = 0.0f;
#pragma unroll
              for (int gr = 0; gr < kG; ++gr) {
                const uint32_t pp = i < 2 ? p0[gr] : p1[gr];
                x = fmaf(par_step(pp), part[gr][nr][i], x);
                y = fmaf(par_min(pp), c_min[nr][i & 1][gr], y);
              }
              sc[mt][nr][i] = fmaf(c_acc[nr][i & 1], x, y);
            }
        }
      }
      Halves ahead;  // the next step
      if constexpr (L::kTwo) {  // K has been read: the next step's K comes in its place
        __syncwarp();
        if ((k + 1) % 16 == 0) look_up(w, k + 1);
        ahead = halves(w, k + 1);
        if (step + kWarps < s_end) copy_k(0, ahead);
        copy_commit();
      } else if constexpr (L::kHalves) {  // the next step's V comes in its place
        __syncwarp();
        if (step + kWarps < s_end) copy_v(k_half, halves(w, k + 1));
        copy_commit();
        if constexpr (!kB) {  // V's pairs come first
          copy_wait<2>();
          __syncwarp();
        }
      }
      // The mask, only where some row of the tile does not see all 32 keys.
      if constexpr (CHOSEN) {
        if (seen_now != 0xffffffffu) {
#pragma unroll
          for (int mt = 0; mt < 2; ++mt)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (!(seen_now >> (mt * 16 + key_at<FMT>(g) + (i >> 1) * 8) & 1u))
#pragma unroll
                for (int nr = 0; nr < NR; ++nr) sc[mt][nr][i] = kNegInf;
        }
      } else if (!(key0 + kRowsStep <= kr.hi_min && (key0 >= kr.lo_max || key0 + kRowsStep <= a.sinks))) {
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int j = key0 + mt * 16 + key_at<FMT>(g) + (i >> 1) * 8;
#pragma unroll
            for (int nr = 0; nr < NR; ++nr) {
              const int h = hi[nr][i & 1];
              const bool sees = j < h && (!a.window || j >= h - a.window || j < a.sinks);
              if (!sees) sc[mt][nr][i] = kNegInf;
            }
          }
      }
      // V's steps and minima of this thread's keys, and room for the largest step.
      float vs[2][2][kG], vm[2][2][kG];
      if constexpr (!kB) {
        uint32_t most = 0;
        uint32_t vp[2][2][kG];
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
          for (int k8 = 0; k8 < 2; ++k8)
#pragma unroll
            for (int gr = 0; gr < kG; ++gr) {
              vp[mt][k8][gr] = lds32(vp_at + ((mt * 16 + key_at<FMT>(g) + 8 * k8) * kG + gr) * 4);
              most = max(most, vp[mt][k8][gr] & 0x7C00u);
            }
        most = min(__reduce_max_sync(0xffffffffu, most) >> 10, 30u);
        if (most > field) {  // rarely: the same for the whole warp
          const float f = __uint_as_float((127u + field - most) << 23);
#pragma unroll
          for (int ct = 0; ct < kCt; ++ct)
#pragma unroll
            for (int nr = 0; nr < NR; ++nr)
#pragma unroll
              for (int i = 0; i < 4; ++i) o[ct][nr][i] *= f;
          field = most;
        }
        const float up = __uint_as_float((127u + 29u - field) << 23);
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
          for (int k8 = 0; k8 < 2; ++k8)
#pragma unroll
            for (int gr = 0; gr < kG; ++gr) {
              vs[mt][k8][gr] = par_step(vp[mt][k8][gr]) * up;
              vm[mt][k8][gr] = par_min(vp[mt][k8][gr]);
            }
      }
      // Softmax: the rows' new maxima, weights, sums
      uint32_t pb[2][NR][2][kB ? 2 : kG];  // bf16: the weight, and what bf16 leaves of it; codes: times each group's step
#pragma unroll
      for (int nr = 0; nr < NR; ++nr) {
        float mx[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          mx[i] = fmaxf(fmaxf(sc[0][nr][i], sc[0][nr][i + 2]), fmaxf(sc[1][nr][i], sc[1][nr][i + 2]));
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], d));
          mx[i] = fmaxf(mx[i], m[nr][i]);
        }
        float f[2], base[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          base[i] = mx[i] == kNegInf ? 0.0f : mx[i];
          f[i] = exp2_fast(m[nr][i] - base[i]);
          m[nr][i] = mx[i];
          l[nr][i] *= f[i];
        }
        if (__any_sync(0xffffffffu, f[0] != 1.0f || f[1] != 1.0f)) {
#pragma unroll
          for (int ct = 0; ct < kCt; ++ct)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[ct][nr][i] *= f[i & 1];
#pragma unroll
          for (int gr = 0; gr < kG; ++gr) pm[nr][0][gr] *= f[0], pm[nr][1][gr] *= f[1];
        }
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
          for (int k8 = 0; k8 < 2; ++k8) {
            const float p0 = exp2_fast(sc[mt][nr][2 * k8] - base[0]), p1 = exp2_fast(sc[mt][nr][2 * k8 + 1] - base[1]);
            l[nr][0] += p0;
            l[nr][1] += p1;
            if constexpr (kB) {
              const uint32_t pk = pack2<true>(p0, p1);
              pb[mt][nr][k8][0] = transpose8(pk);
              pb[mt][nr][k8][1] = transpose8(
                  pack2<true>(p0 - __uint_as_float(pk << 16), p1 - __uint_as_float(pk & 0xFFFF0000u)));
            } else {
#pragma unroll
              for (int gr = 0; gr < kG; ++gr) {
                pb[mt][nr][k8][gr] = transpose8(pack2<false>(p0 * vs[mt][k8][gr], p1 * vs[mt][k8][gr]));
                pm[nr][0][gr] = fmaf(p0, vm[mt][k8][gr], pm[nr][0][gr]);
                pm[nr][1][gr] = fmaf(p1, vm[mt][k8][gr], pm[nr][1][gr]);
              }
            }
          }
      }
      if constexpr (L::kTwo) {
        copy_wait<1>();
        __syncwarp();
      }
      // O^T += V^T P^T
#pragma unroll
      for (int mt = 0; mt < 2; ++mt) {
        if constexpr (kB) {
          const int r = mt * 16 + (lane & 7) + ((lane >> 4) << 3);
#pragma unroll
          for (int ct = 0; ct < kCt; ++ct) {
            uint32_t va[4];
            ldsm4t(va, vs_at + r * R::kRowB + swizzle<FMT, R::kRowB>(r, 2 * ct + ((lane >> 3) & 1)) * 16);
#pragma unroll
            for (int nr = 0; nr < NR; ++nr) {
              mma<true>(o[ct][nr], va, pb[mt][nr][0][0], pb[mt][nr][1][0]);
              mma<true>(o[ct][nr], va, pb[mt][nr][0][1], pb[mt][nr][1][1]);
            }
          }
        } else {
          // Keys of matrix columns 2t, 2t+1, 2t+8, 2t+9
          uint32_t row[4];
          int rk[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            rk[i] = mt * 16 + key_at<FMT>(2 * t + (i & 1)) + (i >> 1) * 8;
            row[i] = vs_at + rk[i] * R::kRowB;
          }
#pragma unroll
          for (int gr = 0; gr < kG; ++gr) {
            constexpr int kW = FMT == kU8 ? 2 : 1;  // words of a group a thread reads
            uint32_t wd[4][kW];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              if constexpr (FMT == kU8) {
                const uint2 x = lds64(row[i] + swizzle<FMT, R::kRowB>(rk[i], gr * 4 + (g >> 1)) * 16 + (g & 1) * 8);
                wd[i][0] = x.x, wd[i][1] = x.y;
              } else {
                wd[i][0] = lds32(row[i] + swizzle<FMT, R::kRowB>(rk[i], gr * 2 + (g >> 2)) * 16 + (g & 3) * 4);
              }
            }
#pragma unroll
            for (int w = 0; w < kW; ++w)
#pragma unroll
              for (int hl = 0; hl < 2; ++hl) {  // lower and upper 16 bits of the words
                const uint32_t e0 = __byte_perm(wd[0][w], wd[1][w], hl ? 0x7632 : 0x5410);
                const uint32_t e1 = __byte_perm(wd[2][w], wd[3][w], hl ? 0x7632 : 0x5410);
                if constexpr (FMT == kU8) {
                  const int ct = gr * 4 + w * 2 + hl;
                  const uint32_t va[4] = {e0 & 0x00FF00FFu, (e0 >> 8) & 0x00FF00FFu, e1 & 0x00FF00FFu, (e1 >> 8) & 0x00FF00FFu};
#pragma unroll
                  for (int nr = 0; nr < NR; ++nr) mma<false>(o[ct][nr], va, pb[mt][nr][0][gr], pb[mt][nr][1][gr]);
                } else {
#pragma unroll
                  for (int q = 0; q < 2; ++q) {  // nibbles 0, 1 and 2, 3 of the 16 bits
                    const int ct = gr * 4 + hl * 2 + q;
                    const uint32_t f0 = e0 >> (8 * q), f1 = e1 >> (8 * q);
                    const uint32_t va[4] = {f0 & 0x000F000Fu, f0 & 0x00F000F0u, f1 & 0x000F000Fu, f1 & 0x00F000F0u};
#pragma unroll
                    for (int nr = 0; nr < NR; ++nr) mma<false>(o[ct][nr], va, pb[mt][nr][0][gr], pb[mt][nr][1][gr]);
                  }
                }
              }
          }
        }
      }
      __syncwarp();  // the stage is read before its next copies are issued
      if constexpr (L::kTwo) {
        if (step + kWarps < s_end) copy_v(1, ahead);
        copy_commit();
        seen_now = ahead.seen;
      } else if constexpr (L::kHalves) {  // K of the step after the next one in V's place
        if ((k + 2) % 16 == 0) look_up(w, k + 2);
        const Halves h = halves(w, k + 2);
        if (step + 2 * kWarps < s_end) copy_k(v_half, h);
        copy_commit();
        seen_now = seen_next, seen_next = h.seen;
        const int free = v_half;
        v_half = k_half, k_half = next_half, next_half = free;
      } else {
        stage = stage + 1 == R::kStages ? 0 : stage + 1;
        if constexpr (CHOSEN) seen_now = seen_next, seen_next = seen_last;
      }
      ++k;
    }
    // The next run's first steps are on their way while this one's results are joined, where these lie elsewhere.
    const bool partial = !(w.starts() && w.ends());
    const int4 record = part_record(w.pair(tiles), head, w.starts(), w.ends());
    go = w.next(a, tiles);
    if (go && !L::kTwo) fill(w);

    // ---- join the warps
    constexpr int kRows = 8 * NR;
    constexpr int kPitch = L::kPitch;
    float* so = reinterpret_cast<float*>(smem + L::kResults);         // [warps][rows][kPitch], warps kApartF apart
    constexpr int kApartF = L::kResultApart / 4;
    float* sm = reinterpret_cast<float*>(smem + L::kStats);           // [warps][rows] maxima, then sums
    float* sl = sm + kWarps * kRows;
#pragma unroll
    for (int nr = 0; nr < NR; ++nr)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float x = l[nr][i];
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
        const int r = nr * 8 + 2 * t + i;
        if (g == 0) {
          sm[warp * kRows + r] = m[nr][i];
          sl[warp * kRows + r] = x;
        }
        float add[kG], times[2] = {1.0f, 1.0f};
#pragma unroll
        for (int gr = 0; gr < kG; ++gr) {
          add[gr] = 0.0f;
          if constexpr (!kB) {
            add[gr] = pm[nr][i][gr];
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) add[gr] += __shfl_xor_sync(0xffffffffu, add[gr], d);
          }
        }
        if constexpr (!kB) {  // codes stood for u 2^-24, odd nibbles for 16 u 2^-24
          times[0] = __uint_as_float((127u + 24u - 29u + field) << 23);
          times[1] = FMT == kU4 ? times[0] * 0.0625f : times[0];
        }
#pragma unroll
        for (int ct = 0; ct < kCt; ++ct)
#pragma unroll
          for (int half = 0; half < 2; ++half)
            so[warp * kApartF + r * kPitch + out_channel<FMT>(ct, half, g)] =
                kB ? o[ct][nr][half * 2 + i] : fmaf(o[ct][nr][half * 2 + i], times[half], add[kB ? 0 : ct >> 2]);
      }
    __syncthreads();
    const int slot = 2 * blockIdx.x + (run > 0 ? 1 : 0);
    if (partial && !clustered) {
      slots |= run > 0 ? 2 : 1;
      if (threadIdx.x == 0) a.part_rec[slot] = record;
    }
    constexpr int kQuads = DP / 4;
    for (int idx = threadIdx.x; idx < kRows * kQuads; idx += kThreads) {
      const int r = idx / kQuads, c = (idx % kQuads) * 4;
      if (row0 + r > row1) continue;
      float top = sm[r];
#pragma unroll
      for (int x = 1; x < kWarps; ++x) top = fmaxf(top, sm[x * kRows + r]);
      const float base = top == kNegInf ? 0.0f : top;
      float sum = 0.0f;
      float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
      for (int x = 0; x < kWarps; ++x) {
        const float f = exp2_fast(sm[x * kRows + r] - base);
        sum += f * sl[x * kRows + r];
        const float4 y = *reinterpret_cast<const float4*>(so + x * kApartF + r * kPitch + c);
        acc.x += f * y.x, acc.y += f * y.y, acc.z += f * y.z, acc.w += f * y.w;
      }
      if (sum == 0.0f) acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);  // sees nothing, here or at all
      if (clustered) {
        float* row = part_rows + r * kPartPitch;
        *reinterpret_cast<float4*>(row + c) = acc;
        if (c == 0) *reinterpret_cast<float2*>(row + DP) = make_float2(top, sum);
      } else if (partial) {
        const int64_t at = static_cast<int64_t>(slot) * kRows + r;
        if (c < a.p.dim) *reinterpret_cast<float4*>(a.part_o + at * a.p.dim + c) = acc;
        if (c == 0) a.part_ml[at] = make_float2(top, sum);
      } else {
        write_row(a, seq, head, row0 + r, c, acc, top, sum);
      }
    }
    __syncthreads();  // the results are read before the next run's are written
    if (go && L::kTwo) fill(w);
  }
  if (clustered) {
    // The cluster's blocks hold a part each, in the place of their rings: every
    // block joins its share of the rows' channels from all of them.
    const Tile x = tile_of<kTileRows, kRowsStep, CHOSEN>(a, tiles, share.p);
    if (share.left <= 0)
      for (int r = threadIdx.x; r < kTileRows; r += kThreads) *reinterpret_cast<float2*>(part_rows + r * kPartPitch + DP) = make_float2(kNegInf, 0.0f);
    cluster_barrier();
    constexpr int kQuads = DP / 4;
    for (int idx = cluster_rank() * kThreads + threadIdx.x; idx < kTileRows * kQuads; idx += a.cluster * kThreads) {
      const int r = idx / kQuads, c = (idx % kQuads) * 4;
      if (r >= x.n_rows) continue;
      const uint32_t row_at = smem_u32(part_rows + r * kPartPitch);
      float2 ml[kCluster];
      float4 y[kCluster];
#pragma unroll
      for (int k = 0; k < kCluster; ++k) ml[k] = k < a.cluster ? far64(in_block(row_at + DP * 4, k)) : make_float2(kNegInf, 0.0f);
#pragma unroll
      for (int k = 0; k < kCluster; ++k)  // a block without steps has left no sums
        y[k] = ml[k].y == 0.0f ? make_float4(0.0f, 0.0f, 0.0f, 0.0f) : far128(in_block(row_at + c * 4, k));
      float top = ml[0].x;
#pragma unroll
      for (int k = 1; k < kCluster; ++k) top = fmaxf(top, ml[k].x);
      const float base = top == kNegInf ? 0.0f : top;
      float sum = 0.0f;
      float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
      for (int k = 0; k < kCluster; ++k) {
        const float f = exp2_fast(ml[k].x - base);
        sum += f * ml[k].y;
        acc.x += f * y[k].x, acc.y += f * y[k].y, acc.z += f * y[k].z, acc.w += f * y[k].w;
      }
      if (sum == 0.0f) acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);  // sees nothing
      write_row(a, x.seq, share.head, x.row0 + r, c, acc, top, sum);
    }
    cluster_barrier();  // a block's shared memory stays until all have read it
  }
  pdl_trigger();
  if (threadIdx.x == 0 && a.unit > 0) {
    if (!(slots & 1)) a.part_rec[2 * blockIdx.x] = make_int4(0, 0, 0, 0);
    if (!(slots & 2)) a.part_rec[2 * blockIdx.x + 1] = make_int4(0, 0, 0, 0);
  }
}

// Joins the parts of a row tile whose keys several blocks shared: a block for
// each block that may start one and each row; a warp takes every fourth part,
// 4 channels per lane, 4 parts at once.
template <int ROWS, bool CHOSEN>
__global__ void __launch_bounds__(kThreads) attend_rows_join_kernel(AttendArgs a, int tiles, int blocks) {
  __shared__ float2 stat[kRowsWarps];
  __shared__ float4 sums[kRowsWarps][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, first = blockIdx.x, r = blockIdx.y, c = lane * 4;
  pdl_trigger();
  pdl_wait();
  int slot;
  int4 rec;
  const int n = parts_from(a, first, blocks, slot, rec);
  if (n == 0) return;
  const Tile x = tile_of<ROWS, kRowsStep, CHOSEN>(a, tiles, rec.y);
  if (r >= x.n_rows) return;
  float top = kNegInf, sum = 0.0f;
  float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  constexpr int kAtOnce = 4;
  for (int i0 = warp; i0 < n; i0 += kRowsWarps * kAtOnce) {
    float2 ml[kAtOnce];
    float4 y[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int i = i0 + k * kRowsWarps;
      const int64_t at = (i == 0 ? slot : 2 * (first + i)) * static_cast<int64_t>(ROWS) + r;
      ml[k] = i < n ? a.part_ml[at] : make_float2(kNegInf, 0.0f);
      y[k] = i < n && c < a.p.dim ? *reinterpret_cast<const float4*>(a.part_o + at * a.p.dim + c) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    }
    float mx = top;
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) mx = fmaxf(mx, ml[k].x);
    const float base = mx == kNegInf ? 0.0f : mx, f0 = exp2_fast(top - base);
    top = mx;
    sum *= f0;
    acc.x *= f0, acc.y *= f0, acc.z *= f0, acc.w *= f0;
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const float f = exp2_fast(ml[k].x - base);
      sum += f * ml[k].y;
      acc.x += f * y[k].x, acc.y += f * y[k].y, acc.z += f * y[k].z, acc.w += f * y[k].w;
    }
  }
  if (lane == 0) stat[warp] = make_float2(top, sum);
  sums[warp][lane] = acc;
  __syncthreads();
  if (warp != 0) return;
#pragma unroll
  for (int k = 1; k < kRowsWarps; ++k) {
    const float2 ml = stat[k];
    const float mx = fmaxf(top, ml.x), base = mx == kNegInf ? 0.0f : mx, f0 = exp2_fast(top - base), f = exp2_fast(ml.x - base);
    const float4 y = sums[k][lane];
    top = mx;
    sum = sum * f0 + f * ml.y;
    acc.x = acc.x * f0 + f * y.x, acc.y = acc.y * f0 + f * y.y, acc.z = acc.z * f0 + f * y.z, acc.w = acc.w * f0 + f * y.w;
  }
  if (sum == 0.0f) acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);  // sees nothing
  write_row(a, x.seq, rec.z, x.row0 + r, c, acc, top, sum);
}

template <int FMT, int DP, int NR, bool CHOSEN>
struct Kernel {
  using L = Layout<FMT, DP, NR, CHOSEN>;
  static constexpr int kSmem = L::kBytes;
  inline static int resident = 0;  // blocks per SM
  static cudaError_t prepare() {
    const cudaError_t e = cudaFuncSetAttribute(attend_rows_kernel<FMT, DP, NR, CHOSEN>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
    if (e != cudaSuccess) return e;
    return cudaOccupancyMaxActiveBlocksPerMultiprocessor(&resident, attend_rows_kernel<FMT, DP, NR, CHOSEN>, kThreads, kSmem);
  }
  static cudaError_t launch(const AttendArgs& a, int blocks, cudaStream_t st) {
    const cudaError_t e =
        launch_clusters(a.unit == 0 ? a.cluster : 1, attend_rows_kernel<FMT, DP, NR, CHOSEN>, dim3(blocks), kThreads, kSmem, st, a, a.tiles);
    if (e != cudaSuccess || a.unit <= 0) return e;
    return launch_next(attend_rows_join_kernel<8 * NR, CHOSEN>, dim3(blocks, 8 * NR), kThreads, 0, st, a, a.tiles, blocks);
  }
};

template <int FMT, bool CHOSEN>
cudaError_t prepare_format() {
  cudaError_t e = Kernel<FMT, 64, 1, CHOSEN>::prepare();
  if (e == cudaSuccess) e = Kernel<FMT, 64, 2, CHOSEN>::prepare();
  if (e == cudaSuccess) e = Kernel<FMT, 128, 1, CHOSEN>::prepare();
  if (e == cudaSuccess) e = Kernel<FMT, 128, 2, CHOSEN>::prepare();
  return e;
}

template <int FMT, bool CHOSEN>
cudaError_t launch_format(const AttendArgs& a, int blocks, cudaStream_t st) {
  if (a.p.dim <= 64)
    return a.tile == 8 ? Kernel<FMT, 64, 1, CHOSEN>::launch(a, blocks, st) : Kernel<FMT, 64, 2, CHOSEN>::launch(a, blocks, st);
  return a.tile == 8 ? Kernel<FMT, 128, 1, CHOSEN>::launch(a, blocks, st) : Kernel<FMT, 128, 2, CHOSEN>::launch(a, blocks, st);
}

template <int FMT, bool CHOSEN>
int resident_format(int dim, int tile) {
  if (dim <= 64) return tile == 8 ? Kernel<FMT, 64, 1, CHOSEN>::resident : Kernel<FMT, 64, 2, CHOSEN>::resident;
  return tile == 8 ? Kernel<FMT, 128, 1, CHOSEN>::resident : Kernel<FMT, 128, 2, CHOSEN>::resident;
}

template <bool CHOSEN>
int resident(int fmt, int dim, int tile) {
  return fmt == kBf16 ? resident_format<kBf16, CHOSEN>(dim, tile)
                      : fmt == kU8 ? resident_format<kU8, CHOSEN>(dim, tile) : resident_format<kU4, CHOSEN>(dim, tile);
}

template <bool CHOSEN>
cudaError_t prepare() {
  cudaError_t e = prepare_format<kBf16, CHOSEN>();
  if (e == cudaSuccess) e = prepare_format<kU8, CHOSEN>();
  if (e == cudaSuccess) e = prepare_format<kU4, CHOSEN>();
  return e;
}

template <bool CHOSEN>
cudaError_t launch(const AttendArgs& a, int blocks, cudaStream_t st) {
  switch (a.p.fmt) {
    case kBf16: return launch_format<kBf16, CHOSEN>(a, blocks, st);
    case kU8: return launch_format<kU8, CHOSEN>(a, blocks, st);
    default: return launch_format<kU4, CHOSEN>(a, blocks, st);
  }
}

}  // namespace

}  // namespace ipv
