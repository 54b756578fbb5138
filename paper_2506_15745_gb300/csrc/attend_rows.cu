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
  static constexpr int kWarp = kStage * kStages;
  static constexpr int kBytes = kWarp * kRowsWarps;
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

// Resident blocks per SM that registers and shared memory are cut to: bf16 at 128
// channels has enough bytes in flight with one, codes need warps to widen them (32
// ragged 4-bit streams: 3 blocks of 168 registers 123 us, 4 of 128, with spills, 134).
constexpr int min_blocks(int fmt, int dp, int nr) { return fmt == kBf16 && dp == 128 ? 1 : nr == 1 ? 3 : 2; }

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

template <int FMT, int DP, int NR>
__global__ void __launch_bounds__(kThreads, min_blocks(FMT, DP, NR)) attend_rows_kernel(AttendArgs a, int tiles) {
  using R = Ring<FMT, DP>;
  constexpr bool kB = FMT == kBf16;
  constexpr int kCh = R::kRowB / 16;     // chunks of a row
  constexpr int kKs = DP / 16;           // k-steps of the first product
  constexpr int kCt = DP / 16;           // channel tiles of the second
  constexpr int kG = kB ? 1 : R::kG;     // accumulators of the first product
  extern __shared__ __align__(128) unsigned char smem[];

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  constexpr int kTileRows = 8 * NR;
  pdl_wait();
  const Share share = find_share<kTileRows, kRowsStep, kRunCost, kThreads>(a, tiles, reinterpret_cast<int64_t*>(smem));
  int slots = 0;  // partial results used
  const bool clustered = a.unit == 0 && a.cluster > 1;
  if (share.left <= 0 && !clustered) {
    if (threadIdx.x < 2 && a.unit > 0) a.part_rec[2 * blockIdx.x + threadIdx.x] = make_int4(0, 0, 0, 0);
    return;
  }
  __syncthreads();  // the shared memory held find_share's scratch
  using W = Walk<kTileRows, kRowsStep, kRunCost>;
  W w = {};
  const uint32_t ring = smem_u32(smem) + warp * R::kWarp;
  const int nch = a.p.row_bytes >> 4;

  // ---- copies of one step into one stage (this warp's lanes only)
  // A lane's chunks are chunk my_c of keys my_r, my_r + 32 / kCh, ...
  constexpr int kApart = 32 / kCh;
  const int my_r = lane / kCh, my_c = lane % kCh;
  const int64_t v_from_k = a.p.v - a.p.k;
  const int64_t page_bytes = a.p.page_stride * a.p.row_bytes, next_bytes = a.p.row_stride * a.p.row_bytes;
  // This lane's key of step i of run x: its page, -1: none. Read a step ahead of
  // the copies.
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
  // The first steps of a run, and the page of the one after them.
  int page_next = -1;
  auto fill = [&](const W& x) {
    int pages[R::kStages];  // all on their way at once
#pragma unroll
    for (int i = 0; i < R::kStages; ++i) pages[i] = page_of(x, x.s + warp + i * kRowsWarps);
#pragma unroll
    for (int i = 0; i < R::kStages - 1; ++i) {
      const int step = x.s + warp + i * kRowsWarps;
      if (step < x.s + x.n) issue(x, step, pages[i], i);
      copy_commit();
    }
    page_next = pages[R::kStages - 1];
  };

  // A cluster's part: [rows][DP sums, maximum, sum] in the rings, which one run leaves free.
  constexpr int kPartPitch = DP + 4;
  float* part_rows = reinterpret_cast<float*>(smem);

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
    for (int step = first; step < s_end; step += kRowsWarps) {
      {
        const int ahead = step + (R::kStages - 1) * kRowsWarps;
        const int to = stage == 0 ? R::kStages - 1 : stage - 1;
        if (ahead < s_end) issue(w, ahead, page_next, to);
        page_next = page_of(w, ahead + kRowsWarps);
        copy_commit();
      }
      copy_wait<R::kStages - 1>();
      __syncwarp();
      const uint32_t ks_at = ring + stage * R::kStage, vs_at = ks_at + R::kTile;
      const uint32_t kp_at = ks_at + 2 * R::kTile, vp_at = kp_at + R::kPar;
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
      // The mask, only where some row of the tile does not see all 32 keys.
      if (!(key0 + kRowsStep <= kr.hi_min && (key0 >= kr.lo_max || key0 + kRowsStep <= a.sinks))) {
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
      stage = stage + 1 == R::kStages ? 0 : stage + 1;
    }
    // The next run's first steps are on their way while this one's results are joined.
    const bool partial = !(w.starts() && w.ends());
    const int4 record = part_record(w.pair(tiles), head, w.starts(), w.ends());
    go = w.next(a, tiles);
    if (go) fill(w);

    // ---- join the warps
    constexpr int kRows = 8 * NR;
    float* so = reinterpret_cast<float*>(smem + R::kBytes);           // [warps][rows][DP + 4]
    constexpr int kPitch = DP + 4;
    float* sm = so + kRowsWarps * kRows * kPitch;                     // [warps][rows] maxima, then sums
    float* sl = sm + kRowsWarps * kRows;
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
            so[(warp * kRows + r) * kPitch + out_channel<FMT>(ct, half, g)] =
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
      for (int x = 1; x < kRowsWarps; ++x) top = fmaxf(top, sm[x * kRows + r]);
      const float base = top == kNegInf ? 0.0f : top;
      float sum = 0.0f;
      float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
      for (int x = 0; x < kRowsWarps; ++x) {
        const float f = exp2_fast(sm[x * kRows + r] - base);
        sum += f * sl[x * kRows + r];
        const float4 y = *reinterpret_cast<const float4*>(so + (x * kRows + r) * kPitch + c);
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
  }
  if (clustered) {
    // The cluster's blocks hold a part each, in the place of their rings: every
    // block joins its share of the rows' channels from all of them.
    const Tile x = tile_of<kTileRows, kRowsStep>(a, tiles, share.p);
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
      for (int k = 0; k < kCluster; ++k) ml[k] = far64(in_block(row_at + DP * 4, k));
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
template <int ROWS>
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
  const Tile x = tile_of<ROWS, kRowsStep>(a, tiles, rec.y);
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

template <int FMT, int DP, int NR>
struct Kernel {
  static constexpr int kSmem = Ring<FMT, DP>::kBytes + kRowsWarps * 8 * NR * (DP + 4 + 2) * 4;  // the rings, the warps' results
  inline static int resident = 0;  // blocks per SM
  static cudaError_t prepare() {
    const cudaError_t e = cudaFuncSetAttribute(attend_rows_kernel<FMT, DP, NR>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
    if (e != cudaSuccess) return e;
    return cudaOccupancyMaxActiveBlocksPerMultiprocessor(&resident, attend_rows_kernel<FMT, DP, NR>, kThreads, kSmem);
  }
  static cudaError_t launch(const AttendArgs& a, int blocks, cudaStream_t st) {
    const cudaError_t e = launch_clusters(a.unit == 0 ? a.cluster : 1, attend_rows_kernel<FMT, DP, NR>, dim3(blocks), kThreads, kSmem, st, a, a.tiles);
    if (e != cudaSuccess || a.unit == 0) return e;
    return launch_next(attend_rows_join_kernel<8 * NR>, dim3(blocks, 8 * NR), kThreads, 0, st, a, a.tiles, blocks);
  }
};

template <int FMT>
cudaError_t prepare_format() {
  cudaError_t e = Kernel<FMT, 64, 1>::prepare();
  if (e == cudaSuccess) e = Kernel<FMT, 64, 2>::prepare();
  if (e == cudaSuccess) e = Kernel<FMT, 128, 1>::prepare();
  if (e == cudaSuccess) e = Kernel<FMT, 128, 2>::prepare();
  return e;
}

template <int FMT>
cudaError_t launch_format(const AttendArgs& a, int blocks, cudaStream_t st) {
  if (a.p.dim <= 64)
    return a.tile == 8 ? Kernel<FMT, 64, 1>::launch(a, blocks, st) : Kernel<FMT, 64, 2>::launch(a, blocks, st);
  return a.tile == 8 ? Kernel<FMT, 128, 1>::launch(a, blocks, st) : Kernel<FMT, 128, 2>::launch(a, blocks, st);
}

template <int FMT>
int resident(int dim, int tile) {
  if (dim <= 64) return tile == 8 ? Kernel<FMT, 64, 1>::resident : Kernel<FMT, 64, 2>::resident;
  return tile == 8 ? Kernel<FMT, 128, 1>::resident : Kernel<FMT, 128, 2>::resident;
}

}  // namespace

int attend_rows_tile(int rows) { return rows <= 8 ? 8 : 16; }

int attend_rows_resident(int fmt, int dim, int tile) {
  return fmt == kBf16 ? resident<kBf16>(dim, tile) : fmt == kU8 ? resident<kU8>(dim, tile) : resident<kU4>(dim, tile);
}

cudaError_t attend_rows_prepare() {
  cudaError_t e = prepare_format<kBf16>();
  if (e == cudaSuccess) e = prepare_format<kU8>();
  if (e == cudaSuccess) e = prepare_format<kU4>();
  return e;
}

cudaError_t launch_attend_rows(const AttendArgs& a, int blocks, cudaStream_t st) {
  switch (a.p.fmt) {
    case kBf16: return launch_format<kBf16>(a, blocks, st);
    case kU8: return launch_format<kU8>(a, blocks, st);
    default: return launch_format<kU4>(a, blocks, st);
  }
}

}  // namespace ipv
