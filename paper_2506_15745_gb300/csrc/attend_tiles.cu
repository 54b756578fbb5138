// Attention of many query rows over a paged cache: chunks of new tokens.
//
// Bound by the tensor cores (4 * head_dim operations per query row and key it
// sees) once there are a few hundred query rows. A block owns 256 query rows
// of one (sequence, KV head): two tiles of 128, in which the query heads that
// share the KV head lie next to each other, so their K and V are fetched once.
// It walks over tiles of 128 keys with ten warps:
//   - one warp copies K and V tiles from their pages by TMA (a box per page),
//   - one thread issues the matrix instructions (tcgen05.mma): S = Q K^T into
//     tensor memory and, with the softmax weights P read from tensor memory,
//     O += P V; while one query tile is in its softmax the other's products run,
//   - a warpgroup per query tile does the softmax, one thread per query row: it
//     reads S, takes exp2, stores P in S's place and keeps the running maximum
//     and sum. O stays in tensor memory and is rescaled only when the maximum
//     has grown by more than 2^8: weights up to 256 are as exact as weights up
//     to 1, and hardly any tile needs it.
// Operands are bf16 (bf16 pages) or fp16 (codes, widened into the workspace
// beforehand); S, O and all statistics are fp32, P is rounded to the operand's
// type.
//
// Tensor memory: S (and P in its place) 2 x 128 columns, O 2 x head_dim.
#include <cuda.h>
#include <cuda_fp16.h>

#include "paged.cuh"

namespace ipv {

// Set when a wait of the kernel below ran out (bit per role); read by
// ipv_attend_error.
__device__ unsigned g_attend_error;

namespace {

constexpr int kRowsCta = kTilesRows;  // query rows of a block
constexpr int kKeys = kTilesStep;     // keys of a step
constexpr int kSoftmaxThreads = 256;
constexpr int kMmaWarp = 8, kLoadWarp = 9;
constexpr int kThreads = 320;
constexpr int kHalf = 128 * 128;      // bytes of 128 rows x 64 channels
constexpr float kNegInf = -INFINITY;
constexpr float kLazy = 8.0f;         // log2 of the growth that rescales O

template <int DP>
struct Layout {
  static constexpr int kHalves = DP / 64;
  static constexpr int kTile = kHalves * kHalf;  // a query, K or V tile
  static constexpr int kStages = DP == 128 ? 2 : 4;
  static constexpr int kQ = 0;
  static constexpr int kK = 2 * kTile;
  static constexpr int kV = kK + kStages * kTile;
  static constexpr int kBars = kV + kStages * kTile;
  static constexpr int kScale = kBars + 256;             // 256 floats
  static constexpr int kBytes = kScale + 1024 + 1024;    // + alignment of the base
};

// Barriers, 8 bytes each.
enum : int { kBarKFull = 0, kBarKEmpty = 4, kBarVFull = 8, kBarVEmpty = 12, kBarS = 16, kBarP = 18, kBarO = 20, kBarQ = 21, kBarDrain = 22,
             kWordTmem = 23 * 8, kWordStop = 24 * 8 };

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

// Waits for a phase of a barrier, at most limit_ns. When the time is up (or
// another warp's was) the block stops: every wait returns false from then on,
// `bit` goes to the error word, and the kernel winds up without results.
__device__ __noinline__ bool bar_wait_slow(uint32_t bar, uint32_t parity, uint32_t stop, int64_t limit_ns, unsigned bit) {
  const uint64_t t0 = now_ns();
  for (;;) {
    if (lds_flag(stop)) return false;
    if (static_cast<int64_t>(now_ns() - t0) >= limit_ns) {
      asm volatile("st.volatile.shared.b32 [%0], %1;" ::"r"(stop), "r"(1u) : "memory");
      atomicOr(&g_attend_error, bit);
      return false;
    }
    for (int i = 0; i < 8; ++i)
      if (bar_try(bar, parity)) return true;
  }
}
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, uint32_t stop, int64_t limit_ns, unsigned bit) {
  if (limit_ns > 0 && bar_try(bar, parity)) return true;
  return bar_wait_slow(bar, parity, stop, limit_ns, bit);
}

__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1, int c2, int c3) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(dst),
      "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3)
      : "memory");
}

__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(acc ? 1u : 0u)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(acc ? 1u : 0u)
      : "memory");
}
__device__ __forceinline__ void mma_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
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
__device__ __forceinline__ void tm_store32(uint32_t at, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};" ::IPV_W8(r, 0),
      IPV_W8(r, 8), IPV_W8(r, 16), IPV_W8(r, 24), "r"(at)
      : "memory");
}
__device__ __forceinline__ void tm_store16(uint32_t at, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};" ::IPV_W8(r, 0),
      IPV_W8(r, 8), "r"(at)
      : "memory");
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

// Shared-memory matrix descriptors, 128-byte swizzle. Rows of 128 bytes, 8 rows
// to an atom of 1024 bytes. K-major (Q, K): atoms 1024 bytes apart along rows.
// MN-major (V: a row is a key, its channels are the instruction's N): atoms
// 1024 bytes apart along keys, 64-channel halves kHalf apart.
__device__ __forceinline__ uint64_t desc_k(uint32_t at) {
  return static_cast<uint64_t>((at & 0x3FFFF) >> 4) | (uint64_t{1} << 16) | (uint64_t{1024 >> 4} << 32) | (uint64_t{1} << 46) |
         (uint64_t{2} << 61);
}
__device__ __forceinline__ uint64_t desc_mn(uint32_t at) {
  return static_cast<uint64_t>((at & 0x3FFFF) >> 4) | (uint64_t{kHalf >> 4} << 16) | (uint64_t{1024 >> 4} << 32) |
         (uint64_t{1} << 46) | (uint64_t{2} << 61);
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
                        int box_rows, int64_t limit_ns) {
  using L = Layout<DP>;
  extern __shared__ unsigned char smem_raw[];
  const int b = blockIdx.z, head = blockIdx.y;
  const int n_tiles = gridDim.x / a.splits;
  // Later tokens see more keys: their blocks start first.
  const int tile = n_tiles - 1 - static_cast<int>(blockIdx.x) / a.splits, split = blockIdx.x % a.splits;
  const Seq seq = sequence(a.p, b);
  const int rows = seq.n * a.share;
  const int row0 = tile * kRowsCta;
  if (row0 >= rows) return;
  const int n_rows = min(kRowsCta, rows - row0);
  const KeyRange kr = key_range(a, seq, row0 / a.share, (row0 + n_rows - 1) / a.share);
  if (split >= splits_of(a, kr)) return;
  const int s_begin = split * a.unit, n = min(kr.steps - s_begin, a.unit);  // steps of this block, maybe 0
  const bool two = n_rows > 128;

  const uint32_t base = (smem_u32(smem_raw) + 1023) & ~1023u;
  unsigned char* base_p = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t bars = base + L::kBars, stop = bars + kWordStop;
  auto bar = [&](int i) { return bars + 8 * i; };
  float* row_scale = reinterpret_cast<float*>(base_p + L::kScale);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(bars + kWordTmem) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  if (threadIdx.x == 0) {
    for (int i = 0; i < 16; ++i) bar_init(bar(i), 1);
    bar_init(bar(kBarS), 1), bar_init(bar(kBarS + 1), 1);
    bar_init(bar(kBarP), 128), bar_init(bar(kBarP + 1), 128);
    bar_init(bar(kBarO), 1), bar_init(bar(kBarDrain), 1);
    bar_init(bar(kBarQ), kSoftmaxThreads);
    asm volatile("st.volatile.shared.b32 [%0], %1;" ::"r"(stop), "r"(0u) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async();
  }
  fence_before();
  __syncthreads();
  fence_after();
  uint32_t tmem;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(tmem) : "r"(bars + kWordTmem) : "memory");

  if (warp == kLoadWarp) {
    // ---------------------------------------------------------------- copies
    const int pieces = kKeys / box_rows;
    const uint32_t piece_bytes = box_rows * 128;
    int issued_k = 0, issued_v = 0;
    bool ok = true;
    for (int i = 0; i < n && ok; ++i) {
      const int st = i % L::kStages;
      const uint32_t empty = ((i / L::kStages) & 1) ^ 1;
      const int key0 = kr.key0(s_begin + i, kKeys);
      const int j = key0 + lane * box_rows;
      const bool active = lane < pieces && j < kr.hi_max;
      int page = 0, row = 0;
      if (active) {
        const int at = j >> a.p.page_shift;
        page = a.p.table ? a.p.table[b * a.p.table_stride + at] : b;
        // A page the pool does not have: past the map's end, which reads as zero.
        if (static_cast<unsigned>(page) >= static_cast<unsigned>(a.p.n_pages)) page = a.p.n_pages;
        row = a.p.page_shift == 31 ? j : j & (a.p.page_size - 1);
      }
      const uint32_t bytes = __popc(__ballot_sync(0xffffffffu, active)) * piece_bytes * L::kHalves;
      for (int kv = 0; kv < 2 && ok; ++kv) {
        const uint32_t full = bar((kv ? kBarVFull : kBarKFull) + st);
        ok = bar_wait(bar((kv ? kBarVEmpty : kBarKEmpty) + st), empty, stop, limit_ns, 1u);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        if (lane == 0) bar_expect(full, bytes);
        __syncwarp();
        if (active) {
          const uint32_t dst = base + (kv ? L::kV : L::kK) + st * L::kTile + lane * piece_bytes;
#pragma unroll
          for (int h = 0; h < L::kHalves; ++h) tma_load(dst + h * kHalf, kv ? &v_map : &k_map, full, 64 * h, row, head, page);
        }
        (kv ? issued_v : issued_k) = i + 1;
        __syncwarp();
      }
    }
    if (!ok) {
      // Stopped: the block's memory must outlive the copies in flight.
      for (int i = max(0, issued_k - L::kStages); i < issued_k; ++i)
        for (int w = 0; w < 1 << 16 && !bar_try(bar(kBarKFull + i % L::kStages), (i / L::kStages) & 1); ++w) {
        }
      for (int i = max(0, issued_v - L::kStages); i < issued_v; ++i)
        for (int w = 0; w < 1 << 16 && !bar_try(bar(kBarVFull + i % L::kStages), (i / L::kStages) & 1); ++w) {
        }
    }
  } else if (warp == kMmaWarp) {
    // -------------------------------------------------------------- products
    const uint32_t idesc_s = instr<BF16>(kKeys, false), idesc_o = instr<BF16>(DP, true);
    bool ok = true;
    auto wait = [&](int i, uint32_t parity, unsigned bit) {
      ok = ok && bar_wait(bar(i), parity, stop, limit_ns, bit);
      ok = __all_sync(0xffffffffu, ok);
      if (ok) fence_after();
      return ok;
    };
    auto scores = [&](int t, int st) {
      if (lane == 0) {
#pragma unroll
        for (int ks = 0; ks < DP / 16; ++ks) {
          const uint32_t off = (ks / 4) * kHalf + (ks % 4) * 32;
          mma_ss(tmem + t * 128, desc_k(base + L::kQ + t * L::kTile + off), desc_k(base + L::kK + st * L::kTile + off), idesc_s,
                 ks > 0);
        }
        mma_commit(bar(kBarS + t));
      }
    };
    auto output = [&](int t, int st, bool acc) {
      if (lane == 0) {
#pragma unroll
        for (int ks = 0; ks < kKeys / 16; ++ks)
          mma_ts(tmem + 256 + t * DP, tmem + t * 128 + ks * 8, desc_mn(base + L::kV + st * L::kTile + ks * 2048), idesc_o,
                 acc || ks > 0);
      }
    };
    if (n > 0) {
      wait(kBarQ, 0, 2u);
      if (ok && wait(kBarKFull, 0, 2u)) {
        scores(0, 0);
        if (two) scores(1, 0);
        if (lane == 0) mma_commit(bar(kBarKEmpty));
      }
    }
    for (int i = 0; i < n && ok; ++i) {
      const int st = i % L::kStages, nx = (i + 1) % L::kStages;
      const bool more = i + 1 < n;
      if (!wait(kBarVFull + st, (i / L::kStages) & 1, 2u)) break;
      const int left = kr.hi_max - kr.key0(s_begin + i, kKeys);
      if (left < kKeys) {
        // Rows past the last key hold anything; a weight of 0 would not hide a NaN.
        for (int x = lane; x < (kKeys - left) * 8 * L::kHalves; x += 32) {
          const int c = x & 7, h = L::kHalves == 2 ? (x >> 3) & 1 : 0, r = left + x / (8 * L::kHalves);
          *reinterpret_cast<uint4*>(base_p + L::kV + st * L::kTile + h * kHalf + r * 128 + c * 16) = make_uint4(0, 0, 0, 0);
        }
        fence_async();
        __syncwarp();
      }
      if (!wait(kBarP, i & 1, 2u)) break;
      output(0, st, i > 0);
      if (more) {
        if (!wait(kBarKFull + nx, ((i + 1) / L::kStages) & 1, 2u)) break;
        scores(0, nx);
      }
      if (two) {
        if (!wait(kBarP + 1, i & 1, 2u)) break;
        output(1, st, i > 0);
        if (more) scores(1, nx);
      }
      if (lane == 0) {
        mma_commit(bar(kBarVEmpty + st));
        if (more) mma_commit(bar(kBarKEmpty + nx));
        if (!more) mma_commit(bar(kBarO));
      }
      __syncwarp();
    }
    if (!ok) {  // stopped: no product may be in flight when the memory goes
      if (lane == 0) mma_commit(bar(kBarDrain));
      for (int w = 0; w < 1 << 16 && !bar_try(bar(kBarDrain), 0); ++w) {
      }
      __syncwarp();
    }
  } else {
    // --------------------------------------------------------------- softmax
    const int t = warp >> 2, wt = threadIdx.x & 127;  // query tile, thread in its warpgroup
    // The query tile into shared memory, swizzled; rows that are not there are zero.
    constexpr int kCh = DP / 8;
    const uint32_t flip = a.scale_log2 < 0.0f ? 0x80008000u : 0u;  // a negative scale turns the queries
    for (int x = wt; x < 128 * kCh; x += 128) {
      const int r = x / kCh, c = x % kCh, rr = t * 128 + r;
      uint4 q = make_uint4(0, 0, 0, 0);
      if (rr < n_rows && c * 8 < a.p.dim) {
        const int tok = (row0 + rr) / a.share, hq = row0 + rr - tok * a.share;
        q = *reinterpret_cast<const uint4*>(a.q + (seq.row0 + static_cast<int64_t>(tok)) * a.q_row +
                                            (head * a.share + hq) * a.q_head + c * 8);
      }
      uint32_t w[4] = {q.x, q.y, q.z, q.w};
      if (BF16) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] ^= flip;
      } else {
        // To fp16: the row's largest magnitude goes to [2^9, 2^10), by a power of two.
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) top = max(top, max(w[i] & 0x7FFFu, (w[i] >> 16) & 0x7FFFu));
#pragma unroll
        for (int d = 1; d < kCh; d <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, d));
        const int e = min(max(static_cast<int>(top >> 7) - 127, -100), 126);
        const float up = __uint_as_float(static_cast<uint32_t>(127 + 9 - e) << 23);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          w[i] ^= flip;
          w[i] = pack2<false>(__uint_as_float(w[i] << 16) * up, __uint_as_float(w[i] & 0xFFFF0000u) * up);
        }
        if (c == 0) row_scale[rr] = fabsf(a.scale_log2) * __uint_as_float(static_cast<uint32_t>(127 - 9 + e) << 23);
      }
      *reinterpret_cast<uint4*>(base_p + L::kQ + t * L::kTile + (c / 8) * kHalf + r * 128 + ((c % 8) ^ (r & 7)) * 16) =
          make_uint4(w[0], w[1], w[2], w[3]);
    }
    fence_async();
    bar_arrive(bar(kBarQ));
    // row_scale: written by this warpgroup's threads, read by others of it
    asm volatile("bar.sync %0, 128;" ::"r"(1 + t) : "memory");

    const int rr = t * 128 + wt;
    const bool in = rr < n_rows;
    const int tok = in ? (row0 + rr) / a.share : 0, hq = in ? head * a.share + row0 + rr - tok * a.share : 0;
    const int hi = in ? token_hi(a, seq, tok) : 0x7FFFFFFF;  // rows that are not there need no mask
    const int lo = in && a.window ? max(0, hi - a.window) : 0;
    // Not 0, which would make a masked score (-inf) NaN.
    const float scale = fmaxf(BF16 ? fabsf(a.scale_log2) : row_scale[rr], 1.17549435e-38f);
    const uint32_t lane_at = tmem + (static_cast<uint32_t>(warp & 3) << 21);
    const uint32_t s_at = lane_at + t * 128, o_at = lane_at + 256 + t * DP;
    float m = kNegInf, l = 0.0f;
    bool ok = true;
    if (t == 0 || two) {
      for (int i = 0; i < n; ++i) {
        ok = __all_sync(0xffffffffu, bar_wait(bar(kBarS + t), i & 1, stop, limit_ns, 4u));
        if (!ok) break;
        fence_after();
        const int key0 = kr.key0(s_begin + i, kKeys);
        uint32_t s[128];
#pragma unroll
        for (int c = 0; c < 4; ++c) tm_load(s + 32 * c, s_at + 32 * c);
        wait_ld();
        const bool all = key0 + kKeys <= hi && (key0 >= lo || key0 + kKeys <= a.sinks);
        if (!__all_sync(0xffffffffu, all)) {
          const int h = hi - key0, w0 = lo - key0, sk = a.sinks - key0;
#pragma unroll
          for (int c = 0; c < 128; ++c)
            if (!(c < h && (c >= w0 || c < sk))) s[c] = 0xFF800000u;
        }
        float mx[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) mx[c] = __uint_as_float(s[c]);
#pragma unroll
        for (int c = 4; c < 128; ++c) mx[c & 3] = fmaxf(mx[c & 3], __uint_as_float(s[c]));
        const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * scale;
        if (__any_sync(0xffffffffu, top > m + kLazy)) {
          const float mn = fmaxf(m, top);
          const float f = mn == kNegInf ? 1.0f : exp2_fast(m - mn);
          m = mn;
          l *= f;
          if (i > 0) {
#pragma unroll
            for (int c = 0; c < DP / 32; ++c) {
              uint32_t o[32];
              tm_load(o, o_at + 32 * c);
              wait_ld();
#pragma unroll
              for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * f);
              tm_store32(o_at + 32 * c, o);
            }
          }
        }
        const float mb = m == kNegInf ? 0.0f : -m;
        const float2 sc2 = make_float2(scale, scale), mb2 = make_float2(mb, mb);
        float2 sum[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint32_t p[16];
#pragma unroll
          for (int k = 0; k < 16; ++k) {
            float2 x = make_float2(__uint_as_float(s[32 * c + 2 * k]), __uint_as_float(s[32 * c + 2 * k + 1]));
            x = fma2(x, sc2, mb2);
            x.x = exp2_fast(x.x);
            x.y = exp2_fast(x.y);
            sum[k & 1] = __fadd2_rn(sum[k & 1], x);
            p[k] = pack2<BF16>(x.x, x.y);
          }
          tm_store16(s_at + 16 * c, p);
        }
        l += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
        wait_st();
        fence_before();
        bar_arrive(bar(kBarP + t));
      }
      if (ok && n > 0) {
        ok = __all_sync(0xffffffffu, bar_wait(bar(kBarO), 0, stop, limit_ns, 4u));
        fence_after();
      }
      if (ok) {
        const int64_t row = seq.row0 + static_cast<int64_t>(tok);
        const int64_t part = (row * a.q_heads + hq) * a.splits + split;
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
        for (int c = 0; c < DP / 32; ++c) {
          uint32_t o[32];
          __syncwarp();
          if (n > 0) {
            tm_load(o, o_at + 32 * c);
            wait_ld();
          }
          if (l == 0.0f) {  // sees nothing, here or at all
#pragma unroll
            for (int k = 0; k < 32; ++k) o[k] = 0u;
          }
          if (in) {
            if (a.splits > 1) {
#pragma unroll
              for (int k = 0; k < 32; k += 4)
                if (32 * c + k < a.p.dim)
                  *reinterpret_cast<uint4*>(a.part_o + part * a.p.dim + 32 * c + k) = make_uint4(o[k], o[k + 1], o[k + 2], o[k + 3]);
            } else {
#pragma unroll
              for (int k = 0; k < 32; k += 8)
                if (32 * c + k < a.p.dim) {
                  uint32_t w[4];
#pragma unroll
                  for (int x = 0; x < 4; ++x)
                    w[x] = pack2<true>(__uint_as_float(o[k + 2 * x]) * inv, __uint_as_float(o[k + 2 * x + 1]) * inv);
                  *reinterpret_cast<uint4*>(a.out + row * a.out_row + hq * a.out_head + 32 * c + k) = make_uint4(w[0], w[1], w[2], w[3]);
                }
            }
          }
        }
        __syncwarp();
        if (in && a.splits > 1) a.part_ml[part] = make_float2(m, l);
        if (in && a.splits == 1 && a.lse) a.lse[row * a.q_heads + hq] = l == 0.0f ? kNegInf : (m + log2f(l)) * 0.6931471805599453f;
      }
    }
  }
  fence_before();
  __syncthreads();
  fence_after();
  if (warp == kMmaWarp) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
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
cudaError_t launch_one(const AttendArgs& a, const CUtensorMap& km, const CUtensorMap& vm, int box_rows, int64_t limit_ns, dim3 grid,
                       cudaStream_t st) {
  attend_tiles_kernel<BF16, DP><<<grid, kThreads, Layout<DP>::kBytes, st>>>(a, km, vm, box_rows, limit_ns);
  return cudaGetLastError();
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

cudaError_t launch_attend_tiles(const AttendArgs& a, bool bf16, const TileMaps& maps, int64_t limit_ns, cudaStream_t st) {
  const int tiles = static_cast<int>((static_cast<int64_t>(a.p.max_rows) * a.share + kRowsCta - 1) / kRowsCta);
  const dim3 grid(static_cast<unsigned>(a.splits) * tiles, static_cast<unsigned>(a.p.heads), static_cast<unsigned>(a.p.n_seqs));
  const CUtensorMap& km = *reinterpret_cast<const CUtensorMap*>(maps.k);
  const CUtensorMap& vm = *reinterpret_cast<const CUtensorMap*>(maps.v);
  if (a.p.dim <= 64)
    return bf16 ? launch_one<true, 64>(a, km, vm, maps.box_rows, limit_ns, grid, st)
                : launch_one<false, 64>(a, km, vm, maps.box_rows, limit_ns, grid, st);
  return bf16 ? launch_one<true, 128>(a, km, vm, maps.box_rows, limit_ns, grid, st)
              : launch_one<false, 128>(a, km, vm, maps.box_rows, limit_ns, grid, st);
}

cudaError_t attend_tiles_error(unsigned* bits) {
  cudaError_t e = cudaDeviceSynchronize();
  if (e == cudaSuccess) e = cudaMemcpyFromSymbol(bits, g_attend_error, sizeof *bits);
  const unsigned zero = 0;
  if (e == cudaSuccess) e = cudaMemcpyToSymbol(g_attend_error, &zero, sizeof zero);
  return e;
}

}  // namespace ipv
