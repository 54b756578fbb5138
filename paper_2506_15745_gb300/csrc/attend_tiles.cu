// Attention of many query rows over a paged cache: chunks of new tokens.
//
// Bound by the tensor cores (4 * head_dim operations per query row and key it
// sees) once there are a few hundred query rows. The unit of work is a step:
// 256 query rows of one (sequence, KV head), as two tiles of 128 in which the
// query heads that share the KV head lie next to each other, by 128 keys. A
// block per SM takes an equal share of all steps, in order; where a share ends
// inside a tile's keys, the block leaves a partial result that a second kernel
// joins. A block has twelve warps:
//   - one copies K tiles from their pages by TMA (a box per page and 64
//     channels), one V tiles: small boxes are slow to issue,
//   - one for each query tile issues its matrix instructions (tcgen05.mma):
//     S = Q K^T into tensor memory and, with the softmax weights P read from
//     tensor memory, O += P V. They take turns, so that one tile's products run
//     while the other is in its softmax; a warp's waits pass during the other's
//     turn,
//   - four for each query tile do its softmax, one thread per query row: it reads
//     S, takes exp2, stores P in S's place and keeps the running maximum and
//     sum. O stays in tensor memory and is rescaled only when the maximum has
//     grown by more than 2^8: weights up to 256 are as exact as weights up to 1,
//     and hardly any step needs it.
// Operands are bf16 (bf16 pages) or fp16 (codes, widened into the workspace
// beforehand); S, O and all statistics are fp32, P is rounded to the operand's
// type.
//
// Tensor memory: S (and P in its place) 2 x 128 columns, O 2 x head_dim.
//
// Measured: 16 frames (3136 tokens, 28 query heads, 4 KV heads, 128 channels) over
// 9408 rows 242 us, 1460 TFLOP/s (77% of the measured bf16 rate; call after call on one
// set of inputs 226); one frame over 6468
// rows 30 us (start, 9 steps per block, join); 8191 tokens under a window of 2000, 16
// query heads of 64 channels, 97 us.
#include <cuda.h>
#include <cuda_fp16.h>

#include "attend_share.cuh"
#include "paged.cuh"

namespace ipv {

// Set when a wait of the kernel below ran out (bit per role); read by
// ipv_attend_error.
__device__ unsigned g_attend_error;

namespace {

constexpr int kRowsCta = kTilesRows;  // query rows of a tile of work
constexpr int kKeys = kTilesStep;     // keys of a step
constexpr int kRunCost = 5;           // what a run of steps costs beside them, in steps
constexpr int kMmaWarp = 8, kLoadWarp = 10;  // warps 8, 9: products of query tiles 0, 1; 10, 11: copies of K, V
constexpr int kThreads = 384;                // two softmax warpgroups, one for copies and products
constexpr int kHalf = 128 * 128;      // bytes of 128 rows x 64 channels
constexpr float kNegInf = -INFINITY;
constexpr float kLazy = 8.0f;         // log2 of the growth that rescales O
constexpr int kAhead = 4;             // pairs between the softmax's pipes

// A warp's results: 32 rows of 32 channels, 16 bytes apart from a multiple of 128.
constexpr int kOutRow = 80, kOutWarp = 32 * kOutRow;

template <int DP>
struct Layout {
  static constexpr int kHalves = DP / 64;
  static constexpr int kTile = kHalves * kHalf;  // a query, K or V tile
  static constexpr int kStages = DP == 128 ? 2 : 4;
  static constexpr int kQ = 0;
  static constexpr int kK = 2 * kTile;
  static constexpr int kV = kK + kStages * kTile;
  static constexpr int kBars = kV + kStages * kTile;
  static constexpr int kScale = kBars + 512;             // 256 floats
  static constexpr int kOut = kScale + 1024;             // results on their way out
  static constexpr int kBytes = kOut + 8 * kOutWarp + 1024;  // + alignment of the base
};

// Barriers, 8 bytes each.
enum : int { kBarKFull = 0, kBarKEmpty = 4, kBarVFull = 8, kBarVEmpty = 12, kBarS = 16, kBarP = 18, kBarO = 22, kBarQ = 24,
             kBarDrain = 26, kBarVTail = 28, kBarTurn = 32, kBars = 34, kWordTmem = 34 * 8, kWordStop = 35 * 8 };

// ------------------------------------------------------------------ PTX
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
  uint32_t done;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(done)
      : "r"(bar), "r"(parity)
      : "memory");
  return done != 0;
}
__device__ __forceinline__ uint64_t now_ns() {
  uint64_t t;
  asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
  return t;
}
__device__ __forceinline__ uint32_t lds_flag(uint32_t at) {
  uint32_t v;
  asm volatile("ld.volatile.shared.b32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
  return v;
}

// Waits for a phase of a barrier, at most limit_ns, with the whole warp. When
// the time is up the block stops: `bit` goes to the error word, every wait
// returns at once from then on, and the kernel winds up without results.
__device__ __forceinline__ void bar_wait_slow(uint32_t bar, uint32_t parity, uint32_t stop, int64_t limit_ns, unsigned bit) {
  const uint64_t t0 = now_ns();
#pragma unroll 1
  for (;;) {
    if (lds_flag(stop)) return;
    if (static_cast<int64_t>(now_ns() - t0) >= limit_ns) {
      asm volatile("st.volatile.shared.b32 [%0], %1;" ::"r"(stop), "r"(1u) : "memory");
      atomicOr(&g_attend_error, bit);
      return;
    }
#pragma unroll 1
    for (int i = 0; i < 8; ++i)
      if (bar_try(bar, parity)) return;
  }
}
// The first try stands in line and the loop out of it: a wait that is over
// costs 60 clocks that way, and 190 where the try is a loop's.
__device__ __forceinline__ void bar_wait(uint32_t bar, uint32_t parity, uint32_t stop, int64_t limit_ns, unsigned bit) {
  bool ok = limit_ns > 0;
  if (ok) ok = bar_try(bar, parity);
  if (__builtin_expect(!ok, 0)) bar_wait_slow(bar, parity, stop, limit_ns, bit);
  __syncwarp();
}

__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1, int c2, int c3) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(dst),
      "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3)
      : "memory");
}

// Shared-memory matrix descriptors, 128-byte swizzle: the low word holds the
// address (in 16 bytes) and the leading offset, the high word the atoms' stride,
// the version and the swizzle. Rows of 128 bytes, 8 rows to an atom of 1024
// bytes. K-major (Q, K): atoms 1024 bytes apart along rows. MN-major (V: a row
// is a key, its channels are the instruction's N): atoms 1024 bytes apart along
// keys, 64-channel halves kHalf apart (the leading offset).
constexpr uint32_t kDescHigh = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint32_t desc_k(uint32_t at) { return ((at & 0x3FFFF) >> 4) | (1u << 16); }
__device__ __forceinline__ uint32_t desc_mn(uint32_t at) { return ((at & 0x3FFFF) >> 4) | (static_cast<uint32_t>(kHalf >> 4) << 16); }

// D (tensor memory) = or += A B, one K = 16 step; OFF: 16-byte units from the
// operands' descriptors (A in tensor memory: columns) to the step's. The whole
// warp runs these and one elected thread issues: operands stay in uniform
// registers, and twice as many instructions wait in the tensor core's queue as
// when a lane issues from a branch of its own.
template <int OFF_A, int OFF_B>
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool acc) {
  asm volatile(
      "{\n\t.reg .pred p, e;\n\t.reg .b32 x, y;\n\t.reg .b64 da, db;\n\t"
      "setp.ne.u32 p, %4, 0;\n\t"
      "add.u32 x, %1, %5;\n\tadd.u32 y, %2, %6;\n\t"
      "mov.b64 da, {x, %7};\n\tmov.b64 db, {y, %7};\n\t"
      "elect.sync _|e, 0xffffffff;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n\t}" ::"r"(d),
      "r"(a), "r"(b), "r"(idesc), "r"(acc ? 1u : 0u), "n"(OFF_A), "n"(OFF_B), "r"(kDescHigh)
      : "memory");
}
template <int OFF_A, int OFF_B>
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool acc) {
  asm volatile(
      "{\n\t.reg .pred p, e;\n\t.reg .b32 x, y;\n\t.reg .b64 db;\n\t"
      "setp.ne.u32 p, %4, 0;\n\t"
      "add.u32 x, %1, %5;\n\tadd.u32 y, %2, %6;\n\t"
      "mov.b64 db, {y, %7};\n\t"
      "elect.sync _|e, 0xffffffff;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [x], db, %3, p;\n\t}" ::"r"(d),
      "r"(a), "r"(b), "r"(idesc), "r"(acc ? 1u : 0u), "n"(OFF_A), "n"(OFF_B), "r"(kDescHigh)
      : "memory");
}
// S = Q K^T (KS steps over the channels) and O += P V (KS over the keys).
template <int KS, int N>
__device__ __forceinline__ void product_s(uint32_t d, uint32_t q, uint32_t k, uint32_t idesc) {
  if constexpr (KS < N) {
    constexpr int kOff = ((KS / 4) * kHalf + (KS % 4) * 32) >> 4;
    mma_ss<kOff, kOff>(d, q, k, idesc, KS > 0);
    product_s<KS + 1, N>(d, q, k, idesc);
  }
}
template <int KS, int N>
__device__ __forceinline__ void product_o(uint32_t d, uint32_t p, uint32_t v, uint32_t idesc, bool acc) {
  if constexpr (KS < N) {
    mma_ts<KS * 8, KS * (2048 >> 4)>(d, p, v, idesc, acc || KS > 0);
    product_o<KS + 1, N>(d, p, v, idesc, acc);
  }
}
__device__ __forceinline__ void mma_commit(uint32_t bar) {  // by the thread that elect.sync elects
  asm volatile(
      "{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t"
      "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar)
      : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

#define IPV_R8(r, o) "=r"(r[o]), "=r"(r[o + 1]), "=r"(r[o + 2]), "=r"(r[o + 3]), "=r"(r[o + 4]), "=r"(r[o + 5]), "=r"(r[o + 6]), "=r"(r[o + 7])
#define IPV_W8(r, o) "r"(r[o]), "r"(r[o + 1]), "r"(r[o + 2]), "r"(r[o + 3]), "r"(r[o + 4]), "r"(r[o + 5]), "r"(r[o + 6]), "r"(r[o + 7])

// 32 columns of the thread's row (lane of tensor memory).
__device__ __forceinline__ void tm_load(uint32_t* r, uint32_t at) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : IPV_R8(r, 0), IPV_R8(r, 8), IPV_R8(r, 16), IPV_R8(r, 24)
      : "r"(at));
}
// Waits for the thread's loads from tensor memory; the registers are those of
// the last one, so that nothing that uses them moves above the wait.
#define IPV_RW8(r, o) "+r"(r[o]), "+r"(r[o + 1]), "+r"(r[o + 2]), "+r"(r[o + 3]), "+r"(r[o + 4]), "+r"(r[o + 5]), "+r"(r[o + 6]), "+r"(r[o + 7])
__device__ __forceinline__ void wait_ld(uint32_t* r) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" : IPV_RW8(r, 0), IPV_RW8(r, 8), IPV_RW8(r, 16), IPV_RW8(r, 24)::"memory");
}
__device__ __forceinline__ void tm_store32(uint32_t at, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};" ::IPV_W8(r, 0),
      IPV_W8(r, 8), IPV_W8(r, 16), IPV_W8(r, 24), "r"(at)
      : "memory");
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void sts128(uint32_t at, const uint32_t (&v)[4]) {
  asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float y;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
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

// Instruction descriptor: fp32 accumulator, both operands bf16 or fp16, M = 128.
template <bool BF16>
__device__ __forceinline__ constexpr uint32_t instr(int n, bool b_mn) {
  return (1u << 4) | ((BF16 ? 1u : 0u) << 7) | ((BF16 ? 1u : 0u) << 10) | ((b_mn ? 1u : 0u) << 16) |
         (static_cast<uint32_t>(n >> 3) << 17) | (static_cast<uint32_t>(128 >> 4) << 24);
}

// ------------------------------------------------------------------ kernel
template <bool BF16, int DP>
__global__ void __launch_bounds__(kThreads, 1)
    attend_tiles_kernel(AttendArgs a, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map,
                        int tiles, int box_rows, int64_t limit_ns) {
  using L = Layout<DP>;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023) & ~1023u;
  unsigned char* base_p = smem_raw + (base - smem_u32(smem_raw));
  pdl_wait();
  const Share share = find_share<kRowsCta, kKeys, kRunCost, kThreads>(a, tiles, reinterpret_cast<int64_t*>(base_p + L::kScale));
  if (share.left <= 0) {
    if (threadIdx.x < 2 && a.unit > 0) a.part_rec[2 * blockIdx.x + threadIdx.x] = make_int4(0, 0, 0, 0);
    return;
  }
  const uint32_t bars = base + L::kBars, stop = bars + kWordStop;
  auto bar = [&](int i) { return bars + 8 * i; };
  float* row_scale = reinterpret_cast<float*>(base_p + L::kScale);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(bars + kWordTmem) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  if (threadIdx.x == 0) {
    for (int i = 0; i < kBars; ++i) {
      const bool tiles2 = (i >= kBarKEmpty && i < kBarVFull) || (i >= kBarVEmpty && i < kBarS);  // both product warps
      const bool warps4 = (i >= kBarP && i < kBarO) || (i >= kBarQ && i < kBarDrain);            // a warpgroup's warps
      bar_init(bar(i), tiles2 ? 2 : warps4 ? 4 : 1);
    }
    asm volatile("st.volatile.shared.b32 [%0], %1;" ::"r"(stop), "r"(0u) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async();
  }
  fence_before();
  __syncthreads();
  fence_after();
  constexpr uint32_t tmem = 0;  // all 512 columns are the block's: they start at 0
  Walk<kRowsCta, kKeys, kRunCost> w = {};

  // Registers: 384 threads start with 168 each; 256 take 224 (a row's 128 scores
  // stay in registers), 128 keep 56: the same 64512 in all.
  if (warp >= kMmaWarp) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    if (warp >= kLoadWarp) {
      // -------------------------------------------------------------- copies
      const bool v = warp > kLoadWarp;
      const CUtensorMap* map = v ? &v_map : &k_map;
      const int full0 = v ? kBarVFull : kBarKFull, empty0 = v ? kBarVEmpty : kBarKEmpty;
      const uint32_t tile0 = base + (v ? L::kV : L::kK);
      const int pieces = kKeys / box_rows;
      const uint32_t piece_bytes = box_rows * 128;
      int it = 0, out = 0;  // steps; tiles asked for
      // This lane's piece of step i: its page and the row there, page < 0: none.
      auto piece = [&](int i, int& page, int& row) {
        const int j = w.t.kr.key0<kKeys>(w.s + i) + lane * box_rows;
        page = -1;
        row = 0;
        if (lane >= pieces || j >= w.t.kr.hi_max) return;
        page = a.p.table ? a.p.table[w.t.b * a.p.table_stride + (j >> a.p.page_shift)] : w.t.b;
        // A page the pool does not have: past the map's end, which reads as zero.
        if (static_cast<unsigned>(page) >= static_cast<unsigned>(a.p.n_pages)) page = a.p.n_pages;
        row = a.p.page_shift == 31 ? j : j & (a.p.page_size - 1);
      };
      for (bool go = w.begin(a, tiles, share); go; go = w.next(a, tiles)) {
        int page_next, row_next;
        piece(0, page_next, row_next);
        for (int i = 0; i < w.n; ++i, ++it) {
          const int st = it % L::kStages, page = page_next, row = row_next;
          const bool active = page >= 0;
          const uint32_t bytes = __popc(__ballot_sync(0xffffffffu, active)) * piece_bytes * L::kHalves;
          if (i + 1 < w.n) piece(i + 1, page_next, row_next);  // the table is read a step ahead
          bar_wait(bar(empty0 + st), ((it / L::kStages) & 1) ^ 1, stop, limit_ns, 1u);
          if (__any_sync(0xffffffffu, lds_flag(stop))) break;
          if (lane == 0) bar_expect(bar(full0 + st), bytes);
          __syncwarp();
          if (active) {
            const uint32_t dst = tile0 + st * L::kTile + lane * piece_bytes;
#pragma unroll
            for (int h = 0; h < L::kHalves; ++h) tma_load(dst + h * kHalf, map, bar(full0 + st), 64 * h, row, w.head, page);
          }
          out = it + 1;
          __syncwarp();
        }
        if (__any_sync(0xffffffffu, lds_flag(stop))) break;
        if (v && w.keep() < kKeys) {
          // Rows past the last key hold anything; a weight of 0 would not hide a NaN.
          const int last = it - 1, st = last % L::kStages, keep = w.keep();
          bar_wait(bar(kBarVFull + st), (last / L::kStages) & 1, stop, limit_ns, 1u);
          for (int x = lane; x < (kKeys - keep) * 8 * L::kHalves; x += 32) {
            const int c = x & 7, h = L::kHalves == 2 ? (x >> 3) & 1 : 0, r = keep + x / (8 * L::kHalves);
            *reinterpret_cast<uint4*>(base_p + L::kV + st * L::kTile + h * kHalf + r * 128 + c * 16) = make_uint4(0, 0, 0, 0);
          }
          fence_async();
          __syncwarp();
          if (lane == 0) bar_arrive(bar(kBarVTail + st));
        }
      }
      if (__any_sync(0xffffffffu, lds_flag(stop))) {
        // Stopped: the block's memory must outlive the copies in flight.
        for (int i = max(0, out - L::kStages); i < out; ++i)
          for (int x = 0; x < 1 << 16 && !bar_try(bar(full0 + i % L::kStages), (i / L::kStages) & 1); ++x) {
          }
      }
    } else {
      // ------------------------------------------------------------ products
      const int t = warp - kMmaWarp;
      constexpr uint32_t idesc_s = instr<BF16>(kKeys, false), idesc_o = instr<BF16>(DP, true);
      const uint32_t q = desc_k(base + L::kQ + t * L::kTile), k0 = desc_k(base + L::kK), v0 = desc_mn(base + L::kV);
      const uint32_t s_at = tmem + t * 128, o_at = tmem + 256 + t * DP;
      auto wait = [&](int i, uint32_t parity) {
        bar_wait(bar(i), parity, stop, limit_ns, 2u);
        fence_after();
      };
      // Scores of step i into S; K's stage is free when they are done.
      auto scores = [&](int i) {
        const int st = i % L::kStages;
        product_s<0, DP / 16>(s_at, q, k0 + st * (L::kTile >> 4), idesc_s);
        mma_commit(bar(kBarS + t));
        mma_commit(bar(kBarKEmpty + st));
      };
      // Turn `it`: tile 0 begins, each tile's end is the other's beginning.
      auto my_turn = [&](int it) { bar_wait(bar(kBarTurn + t), (it & 1) ^ (t == 0 ? 1 : 0), stop, limit_ns, 2u); };
      int it = 0, done = 0, runs = 0;  // steps of the block, of this tile; runs of this tile
      uint32_t tails = 0;              // bit per stage: parity of the tails it has held
      for (bool go = w.begin(a, tiles, share); go; go = w.next(a, tiles)) {
        const bool tail = w.keep() < kKeys;
        if (w.t.n_rows <= 128 * t) {  // no rows in this tile: only lets go of K and V
          for (int i = 0; i < w.n; ++i, ++it) {
            const int st = it % L::kStages;
            wait(kBarKFull + st, (it / L::kStages) & 1);
            if (lane == 0) bar_arrive(bar(kBarKEmpty + st));
            wait(kBarVFull + st, (it / L::kStages) & 1);
            if (lane == 0) bar_arrive(bar(kBarVEmpty + st));
            my_turn(it);
            if (lane == 0) bar_arrive(bar(kBarTurn + (t ^ 1)));
          }
          if (tail) tails ^= 1u << ((it - 1) % L::kStages);
          continue;
        }
        wait(kBarQ + t, runs & 1);
        wait(kBarKFull + it % L::kStages, (it / L::kStages) & 1);
        scores(it);
        for (int i = 0; i < w.n; ++i, ++it, ++done) {
          const int st = it % L::kStages;
          const bool more = i + 1 < w.n;
          if (more || !tail)
            wait(kBarVFull + st, (it / L::kStages) & 1);
          else
            wait(kBarVTail + st, (tails >> st) & 1);
          if (more) wait(kBarKFull + (it + 1) % L::kStages, ((it + 1) / L::kStages) & 1);
          // The weights come in two halves, as the softmax hands them over.
          const uint32_t v = v0 + st * (L::kTile >> 4);
          wait(kBarP + 2 * t, done & 1);
          my_turn(it);
          product_o<0, kKeys / 32>(o_at, s_at, v, idesc_o, i > 0);
          wait(kBarP + 2 * t + 1, done & 1);
          product_o<kKeys / 32, kKeys / 16>(o_at, s_at, v, idesc_o, true);
          if (more) scores(it + 1);
          if (lane == 0) bar_arrive(bar(kBarTurn + (t ^ 1)));
          mma_commit(bar(kBarVEmpty + st));
        }
        mma_commit(bar(kBarO + t));
        if (tail) tails ^= 1u << ((it - 1) % L::kStages);
        ++runs;
      }
      if (__any_sync(0xffffffffu, lds_flag(stop))) {  // stopped: no product may be in flight when the memory goes
        mma_commit(bar(kBarDrain + t));
        for (int x = 0; x < 1 << 16 && !bar_try(bar(kBarDrain + t), 0); ++x) {
        }
        __syncwarp();
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
    // --------------------------------------------------------------- softmax
    const int t = warp >> 2, wt = threadIdx.x & 127;  // query tile, thread in its warpgroup
    const uint32_t lane_at = tmem + (static_cast<uint32_t>(warp & 3) << 21);
    const uint32_t s_at = lane_at + t * 128, o_at = lane_at + 256 + t * DP;
    const uint32_t flip = a.scale_log2 < 0.0f ? 0x80008000u : 0u;  // a negative scale turns the queries
    // A run's query tile into shared memory, swizzled; rows that are not there
    // are zero. A warp loads its own 32 rows. Called when the products that read
    // the tile before it are over.
    auto load_queries = [&](const Walk<kRowsCta, kKeys, kRunCost>& x) {
      if (x.t.n_rows <= 128 * t) return;
      constexpr int kCh = DP / 8, kBatch = 8;
      const int row0 = x.t.row0 + 128 * t, n_rows = x.t.n_rows - 128 * t;
      // The lane's first row and channel; the others follow 32 / kCh rows apart.
      int tok = a.by_share(row0 + 32 * (warp & 3) + lane / kCh);
      int hq = row0 + 32 * (warp & 3) + lane / kCh - tok * a.share;
#pragma unroll 1
      for (int x0 = lane; x0 < 32 * kCh; x0 += 32 * kBatch) {
        uint4 q[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
          const int r = 32 * (warp & 3) + (x0 + 32 * i) / kCh, c = (x0 + 32 * i) % kCh;
          q[i] = make_uint4(0, 0, 0, 0);
          if (r < n_rows && c * 8 < a.p.dim)
            q[i] = *reinterpret_cast<const uint4*>(a.q + (x.t.seq.row0 + static_cast<int64_t>(tok)) * a.q_row +
                                                   (x.head * a.share + hq) * a.q_head + c * 8);
          for (hq += 32 / kCh; hq >= a.share; hq -= a.share) ++tok;
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
          const int r = 32 * (warp & 3) + (x0 + 32 * i) / kCh, c = (x0 + 32 * i) % kCh;
          uint32_t y[4] = {q[i].x, q[i].y, q[i].z, q[i].w};
          if (BF16) {
#pragma unroll
            for (int k = 0; k < 4; ++k) y[k] ^= flip;
          } else {
            // To fp16: the row's largest magnitude goes to [2^9, 2^10), by a power of two.
            uint32_t top = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) top = max(top, max(y[k] & 0x7FFFu, (y[k] >> 16) & 0x7FFFu));
#pragma unroll
            for (int d = 1; d < kCh; d <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, d));
            const int e = min(max(static_cast<int>(top >> 7) - 127, -100), 126);
            const float up = __uint_as_float(static_cast<uint32_t>(127 + 9 - e) << 23);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              y[k] ^= flip;
              y[k] = pack2<false>(__uint_as_float(y[k] << 16) * up, __uint_as_float(y[k] & 0xFFFF0000u) * up);
            }
            if (c == 0) row_scale[128 * t + r] = fabsf(a.scale_log2) * __uint_as_float(static_cast<uint32_t>(127 - 9 + e) << 23);
          }
          *reinterpret_cast<uint4*>(base_p + L::kQ + t * L::kTile + (c / 8) * kHalf + r * 128 + ((c % 8) ^ (r & 7)) * 16) =
              make_uint4(y[0], y[1], y[2], y[3]);
        }
      }
      fence_async();
      __syncwarp();
      if (lane == 0) bar_arrive(bar(kBarQ + t));
    };
    int done = 0, runs = 0, run = 0, slots = 0;  // steps and runs of this tile, of the block; partial results used
    bool go = w.begin(a, tiles, share);
    if (go) load_queries(w);
    while (go) {
      Walk<kRowsCta, kKeys, kRunCost> after = w;
      const bool partial = !(w.starts() && w.ends());
      const int slot = 2 * blockIdx.x + (run > 0 ? 1 : 0);
      ++run;
      if (partial) {
        slots |= slot & 1 ? 2 : 1;
        if (threadIdx.x == 0) a.part_rec[slot] = part_record(w.pair(tiles), w.head, w.starts(), w.ends());
      }
      if (w.t.n_rows <= 128 * t) {
        go = after.next(a, tiles);
        if (go) load_queries(after);
        w = after;
        continue;
      }
      const int row0 = w.t.row0 + 128 * t, n_rows = min(128, w.t.n_rows - 128 * t), head = w.head;
      const bool in = wt < n_rows;
      const int hi = in ? token_hi(a, w.t.seq, a.by_share(row0 + wt)) : 0x7FFFFFFF;  // rows that are not there need no mask
      const int lo = in && a.window ? max(0, hi - a.window) : 0;
      // Not 0, which would make a masked score (-inf) NaN.
      const float scale = fmaxf(BF16 ? fabsf(a.scale_log2) : row_scale[128 * t + wt], 1.17549435e-38f);
      const float2 sc2 = make_float2(scale, scale);
      float m = kNegInf, l = 0.0f;
      for (int i = 0; i < w.n; ++i, ++done) {
        bar_wait(bar(kBarS + t), done & 1, stop, limit_ns, 4u);
        fence_after();
        const int key0 = w.t.kr.key0<kKeys>(w.s + i);
        const bool all = key0 + kKeys <= hi && (key0 >= lo || key0 + kKeys <= a.sinks);
        const bool masked = !__all_sync(0xffffffffu, all);
        const int h = hi - key0, w0 = lo - key0, sk = a.sinks - key0;
        // The weights are taken against the maximum known before this step, and
        // the row's own maximum is found beside them: only if it is more than
        // 2^8 above (hardly ever after the first step) is the first half done again.
        uint32_t s[4][32];
#pragma unroll
        for (int c = 0; c < 4; ++c) tm_load(s[c], s_at + 32 * c);
#pragma unroll
        for (int c = 0; c < 4; ++c) wait_ld(s[c]);
        if (masked) {
          if (__any_sync(0xffffffffu, h < kKeys)) {
#pragma unroll
            for (int c = 0; c < 128; ++c)
              if (c >= h) s[c >> 5][c & 31] = 0xFF800000u;
          }
          if (__any_sync(0xffffffffu, w0 > 0 && sk < kKeys)) {
            const unsigned gap = w0 > sk ? w0 - sk : 0;
#pragma unroll
            for (int c = 0; c < 128; ++c)
              if (static_cast<unsigned>(c - sk) < gap) s[c >> 5][c & 31] = 0xFF800000u;
          }
        }
        float2 mb2, sum[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
        uint32_t p[32];
        float2 x[2 * kAhead];
        // A half row, as 32 pairs: the multiply-add runs kAhead pairs ahead of
        // exp2, the sum and the rounding kAhead behind it, so that no pipe waits.
        auto half = [&](int first, auto also) {
          auto scaled = [&](int k) {
            const uint32_t* y = &s[(first + k) >> 4][2 * ((first + k) & 15)];
            x[k % (2 * kAhead)] = fma2(make_float2(__uint_as_float(y[0]), __uint_as_float(y[1])), sc2, mb2);
          };
          auto weighed = [&](int k) {
            const float2 y = x[k % (2 * kAhead)];
            sum[k & 1] = __fadd2_rn(sum[k & 1], y);
            p[k] = pack2<BF16>(y.x, y.y);
          };
#pragma unroll
          for (int k = 0; k < kAhead; ++k) scaled(k);
#pragma unroll
          for (int k = 0; k < 32; ++k) {
            float2& y = x[k % (2 * kAhead)];
            y.x = exp2_fast(y.x);
            y.y = exp2_fast(y.y);
            also(k);
            if (k >= kAhead) weighed(k - kAhead);
            if (k + kAhead < 32) scaled(k + kAhead);
          }
#pragma unroll
          for (int k = 32 - kAhead; k < 32; ++k) weighed(k);
        };
        auto hand_over = [&](int which) {
          tm_store32(s_at + 32 * which, p);  // in the scores' place: they are all read
          wait_st();
          fence_before();
          __syncwarp();
          if (lane == 0) bar_arrive(bar(kBarP + 2 * t + which));
        };
        auto start = [&]() {
          const float mb = m == kNegInf ? 0.0f : -m;
          mb2 = make_float2(mb, mb);
          sum[0] = sum[1] = make_float2(0.0f, 0.0f);
        };
        float mx[2] = {kNegInf, kNegInf};
        start();
        half(0, [&](int k) {
          mx[0] = max3(mx[0], __uint_as_float(s[k >> 3][(4 * k) & 31]), __uint_as_float(s[k >> 3][(4 * k + 1) & 31]));
          mx[1] = max3(mx[1], __uint_as_float(s[k >> 3][(4 * k + 2) & 31]), __uint_as_float(s[k >> 3][(4 * k + 3) & 31]));
        });
        const float top = fmaxf(mx[0], mx[1]) * scale;
        if (__any_sync(0xffffffffu, top > m + kLazy)) {
          const float mn = fmaxf(m, top);
          const float f = mn == kNegInf ? 1.0f : exp2_fast(m - mn);
          m = mn;
          l *= f;
          if (i > 0) {
#pragma unroll
            for (int c = 0; c < DP / 32; ++c) {
              tm_load(p, o_at + 32 * c);
              wait_ld(p);
#pragma unroll
              for (int k = 0; k < 32; ++k) p[k] = __float_as_uint(__uint_as_float(p[k]) * f);
              tm_store32(o_at + 32 * c, p);
            }
          }
          start();
          half(0, [](int) {});
        }
        hand_over(0);
        half(32, [](int) {});
        hand_over(1);
        l += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
      }
      const int tok = in ? a.by_share(row0 + wt) : 0, hq = in ? head * a.share + row0 + wt - tok * a.share : 0;
      const int64_t row = w.t.seq.row0 + static_cast<int64_t>(tok);
      // The next run's scores are computed while this one's results are written.
      go = after.next(a, tiles);
      if (go) load_queries(after);
      w = after;
      bar_wait(bar(kBarO + t), runs & 1, stop, limit_ns, 4u);
      fence_after();
      ++runs;
      if (__any_sync(0xffffffffu, lds_flag(stop))) break;
      const int64_t part = static_cast<int64_t>(slot) * kRowsCta + 128 * t + wt, out_at = row * a.out_row + hq * a.out_head;
      const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
      for (int c = 0; c < DP / 32; ++c) {
        uint32_t o[32];
        tm_load(o, o_at + 32 * c);
        wait_ld(o);
        if (l == 0.0f) {  // sees nothing, here or at all
#pragma unroll
          for (int k = 0; k < 32; ++k) o[k] = 0u;
        }
        if (partial) {
          // 4 channels of the warp's 32 rows lie next to each other.
          if (in) {
#pragma unroll
            for (int k = 0; k < 32; k += 4)
              if (32 * c + k < a.p.dim)
                *reinterpret_cast<uint4*>(a.part_o + ((static_cast<int64_t>(slot) * (a.p.dim / 4) + 8 * c + k / 4) * kRowsCta + 128 * t + wt) * 4) =
                    make_uint4(o[k], o[k + 1], o[k + 2], o[k + 3]);
          }
        } else {
          // Through shared memory, so that 4 lanes store 64 bytes of a row.
          const uint32_t row_at = base + L::kOut + warp * kOutWarp;
#pragma unroll
          for (int k = 0; k < 32; k += 8) {
            uint32_t y[4];
#pragma unroll
            for (int x = 0; x < 4; ++x)
              y[x] = pack2<true>(__uint_as_float(o[k + 2 * x]) * inv, __uint_as_float(o[k + 2 * x + 1]) * inv);
            sts128(row_at + lane * kOutRow + k * 2, y);
          }
          __syncwarp();
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int r = 8 * k + (lane >> 2), ch = 32 * c + 8 * (lane & 3);
            const uint4 y = lds128(row_at + r * kOutRow + (lane & 3) * 16);
            const int64_t at = __shfl_sync(0xffffffffu, out_at, r);
            if (32 * (warp & 3) + r < n_rows && ch < a.p.dim) *reinterpret_cast<uint4*>(a.out + at + ch) = y;
          }
          __syncwarp();
        }
      }
      __syncwarp();
      if (in && partial) a.part_ml[part] = make_float2(m, l);
      if (in && !partial && a.lse) a.lse[row * a.q_heads + hq] = l == 0.0f ? kNegInf : (m + log2f(l)) * 0.6931471805599453f;
    }
    if (threadIdx.x == 0 && a.unit > 0) {
      if (!(slots & 1)) a.part_rec[2 * blockIdx.x] = make_int4(0, 0, 0, 0);
      if (!(slots & 2)) a.part_rec[2 * blockIdx.x + 1] = make_int4(0, 0, 0, 0);
    }
  }
  pdl_trigger();
  fence_before();
  __syncthreads();
  fence_after();
  // A block that stopped has no parts: thread 0 takes back what it said of them.
  if (threadIdx.x == 0 && a.unit > 0 && lds_flag(stop)) a.part_rec[2 * blockIdx.x] = a.part_rec[2 * blockIdx.x + 1] = make_int4(0, 0, 0, 0);
  if (warp == kMmaWarp) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
}

// Joins the partial results of the tiles that several blocks shared. The block
// where a tile starts holds its first part, the following blocks' first runs the
// others. A block takes 32 query rows, one per lane, and 64 channels, 16 for
// each of its 4 warps; 4 parts at a time are on their way at once.
__global__ void __launch_bounds__(128) attend_tiles_join_kernel(AttendArgs a, int tiles, int blocks) {
  __shared__ __align__(16) uint2 rows[32][17];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x;
  const int r0 = blockIdx.y * 32, r = r0 + lane, quads = a.p.dim / 4, quad0 = 16 * blockIdx.z + 4 * warp;
  pdl_trigger();
  pdl_wait();
  int slot;
  int4 rec;
  const int n = parts_from(a, c, blocks, slot, rec);
  if (n == 0) return;
  const Tile x = tile_of<kRowsCta, kKeys>(a, tiles, rec.y);
  const int n_rows = min(32, x.n_rows - r0);
  if (n_rows <= 0) return;
  float top = kNegInf, sum = 0.0f;
  float4 acc[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) acc[k] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  constexpr int kAtOnce = 4;
  for (int i0 = 0; i0 < n; i0 += kAtOnce) {
    float2 ml[kAtOnce];
    float4 y[kAtOnce][4];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const bool there = i0 + i < n && lane < n_rows;
      const int64_t at = i0 + i == 0 ? slot : 2 * (c + i0 + i);
      ml[i] = there ? a.part_ml[at * kRowsCta + r] : make_float2(kNegInf, 0.0f);
      const float4* o = reinterpret_cast<const float4*>(a.part_o) + (at * quads + quad0) * kRowsCta + r;
#pragma unroll
      for (int k = 0; k < 4; ++k) y[i][k] = there && quad0 + k < quads ? o[k * kRowsCta] : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    }
    float mx = top;
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) mx = fmaxf(mx, ml[i].x);
    const float base = mx == kNegInf ? 0.0f : mx, f0 = exp2_fast(top - base);
    top = mx;
    sum *= f0;
#pragma unroll
    for (int k = 0; k < 4; ++k) acc[k].x *= f0, acc[k].y *= f0, acc[k].z *= f0, acc[k].w *= f0;
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const float f = exp2_fast(ml[i].x - base);
      sum += f * ml[i].y;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        acc[k].x += f * y[i][k].x, acc[k].y += f * y[i][k].y, acc[k].z += f * y[i][k].z, acc[k].w += f * y[i][k].w;
    }
  }
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (sum == 0.0f) acc[k] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);  // sees nothing
    rows[lane][4 * warp + k] = make_uint2(pack2<true>(acc[k].x * inv, acc[k].y * inv), pack2<true>(acc[k].z * inv, acc[k].w * inv));
  }
  __syncthreads();
  const int q = threadIdx.x & 15;  // 16 lanes store 128 bytes of a row
  for (int i = threadIdx.x >> 4; i < n_rows; i += 8) {
    const int tok = a.by_share(x.row0 + r0 + i), hq = rec.z * a.share + x.row0 + r0 + i - tok * a.share;
    const int64_t row = x.seq.row0 + static_cast<int64_t>(tok);
    if (16 * blockIdx.z + q < quads) *reinterpret_cast<uint2*>(a.out + row * a.out_row + hq * a.out_head + 64 * blockIdx.z + 4 * q) = rows[i][q];
  }
  if (warp == 0 && blockIdx.z == 0 && a.lse && lane < n_rows) {
    const int tok = a.by_share(x.row0 + r), hq = rec.z * a.share + x.row0 + r - tok * a.share;
    a.lse[(x.seq.row0 + static_cast<int64_t>(tok)) * a.q_heads + hq] = sum == 0.0f ? kNegInf : (top + log2f(sum)) * 0.6931471805599453f;
  }
}

using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                              const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                              CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeFn g_encode = nullptr;

// A pool of 16-bit rows as (channel, row of a page, head, page); a box is 64
// channels of box_rows rows of one page. False if the map cannot be made.
bool encode(CUtensorMap* map, const Pages& p, const void* base, bool bf16, int box_rows) {
  const int64_t row_b = p.row_bytes;
  auto stride = [&](int64_t s, int64_t count) { return static_cast<cuuint64_t>(count > 1 ? s * row_b : 16); };
  const cuuint64_t dims[4] = {static_cast<cuuint64_t>(p.dim), static_cast<cuuint64_t>(p.page_size),
                              static_cast<cuuint64_t>(p.heads), static_cast<cuuint64_t>(p.n_pages)};
  const cuuint64_t strides[3] = {stride(p.row_stride, p.page_size), stride(p.head_stride, p.heads), stride(p.page_stride, p.n_pages)};
  for (const cuuint64_t s : strides)
    if (s < 16 || s >= (cuuint64_t{1} << 40)) return false;
  const cuuint32_t box[4] = {64, static_cast<cuuint32_t>(box_rows), 1, 1}, one[4] = {1, 1, 1, 1};
  return g_encode(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, const_cast<void*>(base), dims,
                  strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <bool BF16, int DP>
cudaError_t prepare_one() {
  return cudaFuncSetAttribute(attend_tiles_kernel<BF16, DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, Layout<DP>::kBytes);
}

template <bool BF16, int DP>
cudaError_t launch_one(const AttendArgs& a, const CUtensorMap& km, const CUtensorMap& vm, int tiles, int box_rows, int64_t limit_ns,
                       unsigned grid, cudaStream_t st) {
  return launch_next(attend_tiles_kernel<BF16, DP>, dim3(grid), kThreads, Layout<DP>::kBytes, st, a, km, vm, tiles, box_rows, limit_ns);
}

}  // namespace

cudaError_t attend_tiles_prepare() {
  cudaError_t e = prepare_one<true, 64>();
  if (e == cudaSuccess) e = prepare_one<true, 128>();
  if (e == cudaSuccess) e = prepare_one<false, 64>();
  if (e == cudaSuccess) e = prepare_one<false, 128>();
  if (e != cudaSuccess) return e;
  void* fn = nullptr;
  cudaDriverEntryPointQueryResult found;
  e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found);
  if (e != cudaSuccess) return e;
  if (found != cudaDriverEntryPointSuccess) return cudaErrorNotSupported;
  g_encode = reinterpret_cast<EncodeFn>(fn);
  return cudaSuccess;
}

bool attend_tiles_maps(const AttendArgs& a, bool bf16, TileMaps* maps) {
  static_assert(sizeof(CUtensorMap) == sizeof(maps->k) && alignof(TileMaps) % alignof(CUtensorMap) == 0, "tensor map");
  // Pages of fewer rows than a step: a box per page.
  maps->box_rows = a.p.page_size < kKeys ? a.p.page_size : kKeys;
  return encode(reinterpret_cast<CUtensorMap*>(maps->k), a.p, a.p.k, bf16, maps->box_rows) &&
         encode(reinterpret_cast<CUtensorMap*>(maps->v), a.p, a.p.v, bf16, maps->box_rows);
}

cudaError_t launch_attend_tiles(const AttendArgs& a, bool bf16, const TileMaps& maps, int blocks, int64_t limit_ns, cudaStream_t st) {
  const int tiles = a.tiles;
  const CUtensorMap& km = *reinterpret_cast<const CUtensorMap*>(maps.k);
  const CUtensorMap& vm = *reinterpret_cast<const CUtensorMap*>(maps.v);
  cudaError_t e;
  if (a.p.dim <= 64)
    e = bf16 ? launch_one<true, 64>(a, km, vm, tiles, maps.box_rows, limit_ns, blocks, st)
             : launch_one<false, 64>(a, km, vm, tiles, maps.box_rows, limit_ns, blocks, st);
  else
    e = bf16 ? launch_one<true, 128>(a, km, vm, tiles, maps.box_rows, limit_ns, blocks, st)
             : launch_one<false, 128>(a, km, vm, tiles, maps.box_rows, limit_ns, blocks, st);
  if (e != cudaSuccess || a.unit == 0) return e;
  return launch_next(attend_tiles_join_kernel, dim3(blocks, kRowsCta / 32, a.p.dim <= 64 ? 1 : 2), 128, 0, st, a, tiles, blocks);
}

cudaError_t attend_tiles_error(unsigned* bits) {
  cudaError_t e = cudaDeviceSynchronize();
  if (e == cudaSuccess) e = cudaMemcpyFromSymbol(bits, g_attend_error, sizeof *bits);
  const unsigned zero = 0;
  if (e == cudaSuccess) e = cudaMemcpyToSymbol(g_attend_error, &zero, sizeof zero);
  return e;
}

}  // namespace ipv
