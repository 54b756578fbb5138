// Bounds of the keys of pages, and the pages that a query's bounds on them choose.
//
// For each page and KV head, 8-bit integers lo and hi of every channel and one step,
// a power of two, with lo * step <= key <= hi * step for all the page's keys. A query
// row rounded to 8-bit integers qc times a power of two has q . k at most about
// step_q * step * sum over channels of max(qc lo, qc hi), a sum of whole numbers
// below 2^24: exact in any order, so that the pages that are chosen do not depend on
// how the work is split. With q's positive and negative parts kept apart it is a dot
// product, min(qc, 0) . lo + max(qc, 0) . hi, of twice the channels, which the 8-bit
// integer matrix instruction takes: 16 pages by 8 query heads.
#include "paged_codes.cuh"

namespace ipv {
namespace {

constexpr int kLeastExponent = -40;

// The smallest e >= kLeastExponent with m <= 127 * 2^e, m the finite bf16 magnitude
// with these bits (its mantissa of 127 is 127/64 of a power of two).
__device__ __forceinline__ int exponent_of(uint32_t bits) {
  return max(kLeastExponent, static_cast<int>(bits >> 7) - 133 + ((bits & 0x7Fu) == 0x7Fu ? 1 : 0));
}
__device__ __forceinline__ float pow2(int e) { return __uint_as_float(static_cast<uint32_t>(127 + e) << 23); }  // -126 <= e <= 127

__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b) {  // NaN wins
  uint32_t r;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// ------------------------------------------------------------------ the bounds
constexpr int kBoundsThreads = 128;

// The first and last page that hold new rows of a sequence; none: last < first.
__device__ __forceinline__ int2 new_pages(const Pages& p, const Seq& s) {
  if (s.n == 0 || s.len == 0) return make_int2(0, -1);
  return make_int2(max(0, s.len - s.n) >> p.page_shift, (s.len - 1) >> p.page_shift);
}

// The 8-bit bounds of a pair of channels, least and greatest values in bf16; down: 2^-e.
__device__ __forceinline__ uint32_t quantise_pair(uint32_t x, float down, bool upper) {
  uint32_t r = 0;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float y = i ? hi_f(x) : lo_f(x);
    // A product too small for fp32 still lies on its side of 0.
    const int q = upper ? max(static_cast<int>(ceilf(y * down)), y > 0.0f ? 1 : -127) : min(static_cast<int>(floorf(y * down)), y < 0.0f ? -1 : 127);
    r |= (static_cast<uint32_t>(q) & 0xFFu) << (8 * i);
  }
  return r;
}

// A warp takes a page of one head, or four do where pages are long and few. A lane has 16 bytes of a row (8 channels; of codes 16 or
// 32 of one group, in the order in which they are held), 32 / kLanes rows are read at once, kAtOnce times. The minima and maxima
// are taken in bf16 pairs, which codes become first, and then joined by halves: in each round a lane gives away those that
// its partner keeps. The step follows from the largest magnitude's bits.
// A compacted cache of 112 heads of 6272 rows: bf16 (180 MB) 29.4 us, 6.2 TB/s, HBM-bound; 8 bits (96 MB) 28 us, 4 bits 31 us: 7.6
// and 8.3 instructions for each value, with the ALU pipe active 61% and 72% of the time and issue 65% and 64%, at 4 blocks of
// 95 and 124 registers per SM, whose warps wait for their loads between (2.3 and 1.1 of them per issue). A block for each page,
// lanes with 8 channels: 28.8, 53.7 and 49.2 us, and 10.2 instead of 5.0 over 8 x 1000 bf16 rows in pages of 16. bf16, 7 blocks per
// SM: 5 leave a part of a fourth round (30.2 us), 8 spill more than the 8 and 20 bytes of 7 (32.1). Few pages, of 128 rows, 8 x 1000 8-bit rows: 6.6 us with four warps for each, 10.7 with one. The pages of 8 new
// tokens are a launch and three dependent loads.
constexpr int64_t kFewPages = 2048;  // pages and heads up to which four warps take one of more rows than a warp reads at once

// How a lane reads: lanes of a row, rows of a warp, loads at once.
template <int FMT, int G>
struct Lanes {
  static constexpr int kLanes = G * (FMT == kBf16 ? 8 : FMT == kU8 ? 4 : 2), kRows = 32 / kLanes, kAtOnce = FMT == kBf16 ? 8 : 4;
};

// G: groups of 64 channels.
template <int FMT, int G>
__global__ void __launch_bounds__(kBoundsThreads, FMT == kBf16 ? 7 : 4) bounds_kernel(BoundsArgs a, bool together) {
  constexpr int kLanes = Lanes<FMT, G>::kLanes, kRows = Lanes<FMT, G>::kRows, kAtOnce = Lanes<FMT, G>::kAtOnce;
  constexpr int kPairs = FMT == kBf16 ? 4 : FMT == kU8 ? 8 : 16, kAll = kBoundsThreads / 32;
  constexpr int kLeft = kPairs * kLanes / 32;  // pairs that a lane has in the end
  __shared__ uint32_t ends[kAll][2 * kLeft][32];
  pdl_trigger();
  pdl_wait();
  const int b = blockIdx.z, h = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = lane & (kLanes - 1);
  const Seq s = sequence(a.p, b);
  const int2 range = new_pages(a.p, s);
  const int shift = a.p.page_shift, i = range.x + (together ? static_cast<int>(blockIdx.x) : static_cast<int>(blockIdx.x) * kAll + warp);
  if (i > range.y) return;  // together: all warps
  const int pg = a.p.table ? a.p.table[b * a.p.table_stride + i] : b;
  if (static_cast<unsigned>(pg) >= static_cast<unsigned>(a.p.n_pages)) return;
  const bool in = FMT != kBf16 || 8 * c < a.p.dim;
  const int rows = !in ? 0 : shift == 31 ? s.len : min(a.p.page_size, s.len - (i << shift));
  const int64_t row0 = pg * a.p.page_stride + h * a.p.head_stride;
  uint32_t lo[kPairs], hi[kPairs];
#pragma unroll
  for (int k = 0; k < kPairs; ++k) lo[k] = 0x7F807F80u, hi[k] = 0xFF80FF80u;
  for (int r0 = (together ? warp * kRows : 0) + lane / kLanes; r0 < rows; r0 += kRows * kAtOnce * (together ? kAll : 1)) {
    uint4 x[kAtOnce];
    uint32_t par[kAtOnce];
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      const int r = r0 + u * kRows * (together ? kAll : 1);
      if (r >= rows) continue;
      const int64_t row = row0 + r * a.p.row_stride;
      x[u] = ld_once(a.p.k + row * a.p.row_bytes + 16 * c);
      if (FMT != kBf16) par[u] = a.p.k_par[row * G + c / (kLanes / G)];
    }
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      if (r0 + u * kRows * (together ? kAll : 1) >= rows) continue;
      const uint32_t ws[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
#pragma unroll
      for (int j = 0; j < kPairs / 4; ++j) {
        const uint32_t w[2] = {ws[FMT == kU8 ? 2 * j : j], ws[FMT == kU8 ? 2 * j + 1 : j]};
        const uint4 y = FMT == kBf16 ? x[u] : expand<FMT == kBf16 ? kU8 : FMT, false>(w, par[u]);
        const uint32_t ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) lo[4 * j + k] = min_bf16x2(lo[4 * j + k], ys[k]), hi[4 * j + k] = max_bf16x2(hi[4 * j + k], ys[k]);
      }
    }
  }
  int first = 0;  // of the pairs that this lane keeps
#pragma unroll
  for (int d = 16, half = kPairs / 2; d >= kLanes; d >>= 1, half >>= 1) {
    const bool upper = lane & d;
    if (upper) first += half;
#pragma unroll
    for (int k = 0; k < half; ++k) {
      const uint32_t l = __shfl_xor_sync(0xffffffffu, upper ? lo[k] : lo[k + half], d), g = __shfl_xor_sync(0xffffffffu, upper ? hi[k] : hi[k + half], d);
      lo[k] = min_bf16x2(upper ? lo[k + half] : lo[k], l);
      hi[k] = max_bf16x2(upper ? hi[k + half] : hi[k], g);
    }
  }
  if (together) {
#pragma unroll
    for (int k = 0; k < kLeft; ++k) ends[warp][2 * k][lane] = lo[k], ends[warp][2 * k + 1][lane] = hi[k];
    __syncthreads();
    if (warp > 0) return;
#pragma unroll
    for (int w = 1; w < kAll; ++w)
#pragma unroll
      for (int k = 0; k < kLeft; ++k) lo[k] = min_bf16x2(lo[k], ends[w][2 * k][lane]), hi[k] = max_bf16x2(hi[k], ends[w][2 * k + 1][lane]);
  }
  uint32_t top = 0;
#pragma unroll
  for (int k = 0; k < kLeft && in; ++k)
    top = max(max(max(top, lo[k] & 0x7FFFu), max((lo[k] >> 16) & 0x7FFFu, hi[k] & 0x7FFFu)), (hi[k] >> 16) & 0x7FFFu);
  top = __reduce_max_sync(0xffffffffu, top);
  const bool finite = top < 0x7F80u;
  const int e = finite ? exponent_of(top) : 0;
  const int64_t at = static_cast<int64_t>(pg) * a.p.heads + h;
  char* out = a.codes + at * 2 * a.padded;
#pragma unroll
  for (int k = 0; k < kLeft; ++k) {
    // Pair n of chunk q of a group. Codes: words g hold 4 (8 bits) or 8 channels from 4 g or 8 g on, and stand in the places that
    // place_u8 and place_u4 give.
    const int n = first + k, q = c & (kLanes / G - 1), j = FMT == kU8 ? n >> 1 : n >> 2;
    const int channel = c / (kLanes / G) * kGroup + (FMT == kBf16 ? 8 * q + 2 * n
                                                     : FMT == kU8 ? 4 * (q + 4 * j) + 2 * (n & 1)
                                                                  : 8 * (2 * q + (j >> 1) + 4 * (j & 1)) + 2 * (n & 3));
    const bool some = finite && in;  // the padding is 0
    const uint32_t below = some ? quantise_pair(lo[k], pow2(-e), false) : 0u, above = some ? quantise_pair(hi[k], pow2(-e), true) : 0u;
    *reinterpret_cast<uint16_t*>(out + channel) = static_cast<uint16_t>(below);
    *reinterpret_cast<uint16_t*>(out + a.padded + channel) = static_cast<uint16_t>(above);
  }
  if (lane == 0) a.steps[at] = finite ? pow2(e) : __uint_as_float(0x7FC00000u);
}

// ------------------------------------------------------------------ the choice
constexpr int kWarps = kChooseThreads / 32;
constexpr int kBins = 256;      // of the search for the last page that is chosen
static_assert(kBins == kChooseThreads, "a thread has a bin, and a candidate");

__device__ __forceinline__ void mma_s8(int (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint4 lds_u4(const unsigned char* p) { return *reinterpret_cast<const uint4*>(p); }

// Scores as unsigned numbers in the same order; NaN is below all of them.
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t b = __float_as_uint(x);
  return isnan(x) ? 0u : b & 0x80000000u ? ~b : b | 0x80000000u;
}

__device__ __forceinline__ uint32_t rank_in_cluster() {
  uint32_t r;
  asm volatile("mov.u32 %0, %cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void store_in_first(uint32_t at, uint32_t x) {  // into block 0 of the cluster
  uint32_t far;
  asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(far) : "r"(at));
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(far), "r"(x) : "memory");
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// Sum over the block's threads before this one, and over all; scratch: a word per warp.
__device__ __forceinline__ int before_me(int x, int* scratch, int& all) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int upto = x;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, upto, d);
    if (lane >= d) upto += y;
  }
  __syncthreads();  // scratch has been read
  if (lane == 31) scratch[warp] = upto;
  __syncthreads();
  int before = upto - x;
  all = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    const int y = scratch[w];
    if (w < warp) before += y;
    all += y;
  }
  return before;
}

// How many of keys[from..upto) are above k; unrolled, for latency.
__device__ __forceinline__ int count_above(const uint32_t* keys, int from, int upto, uint32_t k) {
  int n = 0;
#pragma unroll 8
  for (int i = from; i < upto; ++i) n += keys[i] > k;
  return n;
}

// Of keys[first..end) the `need` largest, ties to the lower index, get the key
// 0xFFFFFFFF; the others keep theirs. Returns what the chosen keys are above. 0 < need < end - first.
// Up to a key per thread each is ranked among all. Else rounds of a histogram over equal ranges
// of keys narrow [lo, hi] to the range in which the last chosen key lies until a thread
// can rank each that is in it, or it is one key: every round leaves 1/256 of the range, so
// there are 4 at most.
__device__ uint32_t mark_largest(uint32_t* keys, int first, int end, int need, int* bins, uint32_t* cand, int* scratch) {
  int inside = end - first;
  if (inside <= kChooseThreads) {
    const int p = first + static_cast<int>(threadIdx.x);
    const uint32_t k = p < end ? keys[p] : 0u;
    // Equal keys before p come first: there, above k - 1 (k = 0: all).
    const int before = p < end ? (k ? count_above(keys, first, p, k - 1) : p - first) + count_above(keys, p + 1, end, k) : need;
    __syncthreads();
    if (before < need) keys[p] = 0xFFFFFFFFu;
    __syncthreads();
    return 0xFFFFFFFEu;
  }
  uint32_t lo = 0xFFFFFFFFu, hi = 0;
  for (int p = first + threadIdx.x; p < end; p += kChooseThreads) lo = min(lo, keys[p]), hi = max(hi, keys[p]);
  lo = __reduce_min_sync(0xffffffffu, lo);
  hi = __reduce_max_sync(0xffffffffu, hi);
  if ((threadIdx.x & 31) == 0) cand[threadIdx.x >> 5] = lo, cand[kWarps + (threadIdx.x >> 5)] = hi;
  bins[threadIdx.x] = 0;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWarps; ++w) lo = min(lo, cand[w]), hi = max(hi, cand[kWarps + w]);
  while (inside > kChooseThreads && lo < hi) {  // bins are clear; `need` of the `inside` keys in lo..hi are wanted, and all above
    const int shift = max(0, 24 - __clz(hi - lo));  // bins of 2^shift keys, 256 of them reach
    for (int p = first + threadIdx.x; p < end; p += kChooseThreads) {
      const uint32_t k = keys[p];
      if (k >= lo && k <= hi) atomicAdd(bins + ((hi - k) >> shift), 1);  // bin 0 has the largest
    }
    __syncthreads();
    const int mine = bins[threadIdx.x];
    bins[threadIdx.x] = 0;
    int all;
    const int above = before_me(mine, scratch, all);
    if (above < need && above + mine >= need) {
      const uint32_t top = hi - (static_cast<uint32_t>(threadIdx.x) << shift), width = (1u << shift) - 1;
      cand[0] = top;
      cand[1] = top - lo < width ? lo : top - width;
      cand[2] = static_cast<uint32_t>(need - above);
      cand[3] = static_cast<uint32_t>(mine);
    }
    __syncthreads();
    hi = cand[0], lo = cand[1], need = static_cast<int>(cand[2]), inside = static_cast<int>(cand[3]);
    __syncthreads();
  }
  if (inside <= kChooseThreads) {
    if (threadIdx.x == 0) scratch[kWarps] = 0;
    __syncthreads();
    uint32_t* index = cand + kChooseThreads;
    for (int p = first + threadIdx.x; p < end; p += kChooseThreads) {
      const uint32_t k = keys[p];
      if (k >= lo && k <= hi) {
        const int at = atomicAdd(scratch + kWarps, 1);  // in any order: ranks go by key and index
        cand[at] = k, index[at] = static_cast<uint32_t>(p);
      }
    }
    __syncthreads();
    if (static_cast<int>(threadIdx.x) < inside) {
      const uint32_t k = cand[threadIdx.x], p = index[threadIdx.x];
      int before = 0;
#pragma unroll 4
      for (int i = 0; i < inside; ++i) before += cand[i] > k || (cand[i] == k && index[i] < p);
      if (before < need) keys[p] = 0xFFFFFFFFu;
    }
  } else {  // more equal keys than threads: the first `need` of them, in order
    for (int p0 = first; p0 < end && need > 0; p0 += kChooseThreads) {
      const int p = p0 + static_cast<int>(threadIdx.x);
      const bool is = p < end && keys[p] == hi;
      int all;
      const int at = before_me(is ? 1 : 0, scratch, all);
      if (is && at < need) keys[p] = 0xFFFFFFFFu;
      need -= all;
    }
  }
  __syncthreads();
  return hi;
}

// A cluster takes one new row and KV head: its blocks score the pages, 16 at a time
// per warp, the next 16 on their way, into the first block's shared memory; that block chooses. Every
// page's 2 dim + 4 bytes are read once for a row, by the rows of a question each for itself (8 ragged streams of up to 61 rows,
// 193 pages, 4 KV heads: 30 us for 3.4 MB of bounds and queries). 32 ragged streams of up to 769 pages, 8 KV heads with 8 query
// heads each (31 MB): 14.5 us, 2.1 TB/s. The longest streams' blocks set the time, one for each list: 7 rounds per warp of loads, products and
// maxima, one after the other, then the selection with its barriers (2.5 us); without the products 2.4 us less. Issue is active
// 24%: latency, and not of the loads alone, as rings of 3 tiles in shared memory (asynchronous copies) were no faster (14.4 us, of
// equally long streams 18.2 against 15.8), nor were more warps per list (512 threads: 15.1 us, spills; at 256 the kernel for 128
// channels spills 4 bytes) or four blocks per SM (64 registers: 30 us). One stream, 98 pages: 4.8 us.
template <int DP>
__global__ void __launch_bounds__(kChooseThreads, 2) choose_kernel(ChooseArgs a) {
  constexpr int kCodes = 2 * DP;              // bytes of a page's bounds, and of a query head's parts
  constexpr int kVectors = kCodes / 64;       // 16-byte vectors of a row per thread of a quad
  extern __shared__ __align__(16) unsigned char smem[];
  unsigned char* parts = smem;                                              // [head tiles][8][kCodes]
  float* up = reinterpret_cast<float*>(smem + a.head_tiles * 8 * kCodes);   // [head tiles][8]
  uint32_t* cand = reinterpret_cast<uint32_t*>(up + a.head_tiles * 8);      // [threads][2]
  int* bins = reinterpret_cast<int*>(cand + 2 * kChooseThreads);            // [kBins]
  int* scratch = bins + kBins;                                              // [kWarps + 1], rounded up
  uint32_t* keys = reinterpret_cast<uint32_t*>(scratch + 16);               // [pages]
  const int b = blockIdx.z, h = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const int token = static_cast<int>(blockIdx.x) / a.cluster, rank = a.cluster > 1 ? static_cast<int>(rank_in_cluster()) : 0;
  if (a.cluster > 1) cluster_arrive();  // all of them are there before one writes to another
  pdl_trigger();
  pdl_wait();
  // A warp's tiles of 16 pages, and lane i < 16 of it page i's place in the pool: looked up a tile ahead, the first
  // before the sequence's length is known.
  const int stride = a.cluster * kWarps * 16;
  auto look_up = [&](int p0) {
    const int p = p0 + lane;
    int pg = -1;
    if (lane < 16 && p < a.max_pages) pg = a.p.table ? a.p.table[b * a.p.table_stride + p] : b;
    return static_cast<unsigned>(pg) < static_cast<unsigned>(a.p.n_pages) ? pg : -1;
  };
  int p0 = (rank * kWarps + warp) * 16;
  int pg = look_up(p0);
  const Seq s = sequence(a.p, b);
  const bool there = token < s.n;
  const int pos = s.len - s.n + token;
  const int pages = there && pos >= 0 ? (pos >> a.p.page_shift) + 1 : 0;
  const int64_t row = s.row0 + static_cast<int64_t>(token);
  int32_t* out = a.out + row * a.out_row + h * a.out_head;
  const bool all = pages <= a.n;  // nothing to choose
  const float none = __uint_as_float(0x7FC00000u);
  // Lane (g, t) has the 16-byte vectors t, t + 4, .. of pages g and g + 8 of a tile, which stand for
  // four k-steps' operands; the query parts are read in the same order.
  struct Bounds {
    uint4 a[kVectors], b[kVectors];
    float step_a, step_b;
  };
  auto fetch = [&](Bounds& x, int pg) {
    const int pa = __shfl_sync(0xffffffffu, pg, g), pb = __shfl_sync(0xffffffffu, pg, g + 8);
    const char* ca = a.codes + (static_cast<int64_t>(pa) * a.p.heads + h) * kCodes + 16 * t;
    const char* cb = a.codes + (static_cast<int64_t>(pb) * a.p.heads + h) * kCodes + 16 * t;
#pragma unroll
    for (int v = 0; v < kVectors; ++v) {
      x.a[v] = x.b[v] = make_uint4(0, 0, 0, 0);
      if (pa >= 0) x.a[v] = ld_once(ca + 64 * v);
      if (pb >= 0) x.b[v] = ld_once(cb + 64 * v);
    }
    x.step_a = pa >= 0 ? a.steps[static_cast<int64_t>(pa) * a.p.heads + h] : none;
    x.step_b = pb >= 0 ? a.steps[static_cast<int64_t>(pb) * a.p.heads + h] : none;
  };
  Bounds now;
  if (!all) {
    if (p0 < pages) {
      fetch(now, pg);
      pg = look_up(p0 + stride);
    }
    // ---- the query heads, 4 or 2 channels per lane
    constexpr int kLane = DP / 32;
    for (int q = warp; q < a.head_tiles * 8; q += kWarps) {
      uint32_t bits[kLane] = {};
      if (q < a.share && lane * kLane < a.p.dim) {
        const uint16_t* x = a.q + row * a.q_row + static_cast<int64_t>(h * a.share + q) * a.q_head + lane * kLane;
        const uint32_t w = *reinterpret_cast<const uint32_t*>(x);
        bits[0] = w & 0xFFFFu, bits[1] = w >> 16;
        if constexpr (kLane == 4) {
          const uint32_t w2 = *reinterpret_cast<const uint32_t*>(x + 2);
          bits[2] = w2 & 0xFFFFu, bits[3] = w2 >> 16;
        }
      }
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < kLane; ++i) top = max(top, bits[i] & 0x7FFFu);
      top = __reduce_max_sync(0xffffffffu, top);
      const bool counts = q < a.share && top < 0x7F80u;
      const int e = counts ? exponent_of(top) : 0;
      uint32_t neg = 0, plus = 0;
#pragma unroll
      for (int i = 0; i < kLane; ++i) {
        const int x = counts ? __float2int_rn(__uint_as_float(bits[i] << 16) * pow2(-e)) : 0;
        neg |= (static_cast<uint32_t>(min(x, 0)) & 0xFFu) << (8 * i);
        plus |= (static_cast<uint32_t>(max(x, 0)) & 0xFFu) << (8 * i);
      }
      unsigned char* to = parts + q * kCodes + lane * kLane;
      if constexpr (kLane == 4) {
        *reinterpret_cast<uint32_t*>(to) = neg;
        *reinterpret_cast<uint32_t*>(to + DP) = plus;
      } else {
        *reinterpret_cast<uint16_t*>(to) = static_cast<uint16_t>(neg);
        *reinterpret_cast<uint16_t*>(to + DP) = static_cast<uint16_t>(plus);
      }
      if (lane == 0) up[q] = counts ? pow2(e) : none;
    }
  }
  __syncthreads();
  if (a.cluster > 1) cluster_wait();
  if (!all) {
    // ---- scores, the next tile's bounds on their way
    const uint32_t keys_at = smem_u32(keys);
    for (; p0 < pages; p0 += stride) {
      Bounds next;
      if (p0 + stride < pages) {
        fetch(next, pg);
        pg = look_up(p0 + 2 * stride);
      }
      float best_a = none, best_b = none;
      for (int ht = 0; ht < a.head_tiles; ++ht) {
        int parts_c[kVectors][4] = {};  // sums apart: a matrix instruction does not wait for the one before
        const unsigned char* at = parts + (ht * 8 + g) * kCodes + 16 * t;
#pragma unroll
        for (int v = 0; v < kVectors; ++v) {
          const uint4 q = lds_u4(at + 64 * v);
          mma_s8(parts_c[v], now.a[v].x, now.b[v].x, now.a[v].y, now.b[v].y, q.x, q.y);
          mma_s8(parts_c[v], now.a[v].z, now.b[v].z, now.a[v].w, now.b[v].w, q.z, q.w);
        }
        int c[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          c[i] = parts_c[0][i] + parts_c[1][i];
          if constexpr (kVectors == 4) c[i] += parts_c[2][i] + parts_c[3][i];
        }
        const float2 u = *reinterpret_cast<const float2*>(up + ht * 8 + 2 * t);
        best_a = fmaxf(best_a, fmaxf(static_cast<float>(c[0]) * u.x * now.step_a, static_cast<float>(c[1]) * u.y * now.step_a));  // NaN loses
        best_b = fmaxf(best_b, fmaxf(static_cast<float>(c[2]) * u.x * now.step_b, static_cast<float>(c[3]) * u.y * now.step_b));
      }
#pragma unroll
      for (int d = 1; d < 4; d <<= 1) {
        best_a = fmaxf(best_a, __shfl_xor_sync(0xffffffffu, best_a, d));
        best_b = fmaxf(best_b, __shfl_xor_sync(0xffffffffu, best_b, d));
      }
      const int p = p0 + g + 8 * t;
      if (t < 2 && p < pages) {
        const uint32_t k = order_of(t == 0 ? best_a : best_b);
        if (a.cluster > 1)
          store_in_first(keys_at + 4 * p, k);
        else
          keys[p] = k;
      }
      now = next;
    }
  }
  if (a.cluster > 1) {
    cluster_arrive();
    cluster_wait();
  }
  if (!there || rank != 0) return;
  if (all) {
    for (int i = threadIdx.x; i < a.n; i += kChooseThreads) out[i] = i < pages ? i : -1;
    return;
  }
  __syncthreads();
  const int need = a.n - a.first - a.recent, end = pages - a.recent;
  const uint32_t least = need > 0 ? mark_largest(keys, a.first, end, need, bins, cand, scratch) : 0u;
  // ---- the list, in order: a thread has a run of pages
  const int per = (pages + kChooseThreads - 1) / kChooseThreads, from = threadIdx.x * per, upto = min(pages, from + per);
  auto chosen = [&](int p) { return p < a.first || p >= end || (need > 0 && keys[p] > least); };
  int count = 0;
  for (int p = from; p < upto; ++p) count += chosen(p);
  int total;
  int at = before_me(count, scratch, total);
  for (int p = from; p < upto; ++p)
    if (chosen(p)) out[at++] = p;
}

template <int DP>
size_t choose_smem(int head_tiles, int pages) {
  return static_cast<size_t>(head_tiles) * 8 * (2 * DP + 4) + 8 * kChooseThreads + 4 * kBins + 64 + 4 * static_cast<size_t>(pages);
}

}  // namespace

namespace {

template <int FMT, int G>
cudaError_t launch_format(const BoundsArgs& a, int pages, cudaStream_t st) {
  constexpr int kApart = kBoundsThreads / 32;
  const bool together = a.p.page_size > Lanes<FMT, G>::kRows * Lanes<FMT, G>::kAtOnce && static_cast<int64_t>(pages) * a.p.heads * a.p.n_seqs <= kFewPages;
  const dim3 g(static_cast<unsigned>(together ? pages : (pages + kApart - 1) / kApart), static_cast<unsigned>(a.p.heads),
               static_cast<unsigned>(a.p.n_seqs));
  return launch_next(bounds_kernel<FMT, G>, g, kBoundsThreads, 0, st, a, together);
}

template <int FMT>
cudaError_t launch_format(const BoundsArgs& a, int pages, cudaStream_t st) {
  return a.p.groups == 1 ? launch_format<FMT, 1>(a, pages, st) : launch_format<FMT, 2>(a, pages, st);
}

}  // namespace

cudaError_t launch_bounds(const BoundsArgs& a, int pages, cudaStream_t st) {
  switch (a.p.fmt) {
    case kBf16: return launch_format<kBf16>(a, pages, st);
    case kU8: return launch_format<kU8>(a, pages, st);
    default: return launch_format<kU4>(a, pages, st);
  }
}

cudaError_t choose_prepare() {
  cudaError_t e = cudaFuncSetAttribute(choose_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, kChooseSmem);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(choose_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, kChooseSmem);
  return e;
}

cudaError_t launch_choose(const ChooseArgs& a, int pages, cudaStream_t st) {
  const dim3 g(static_cast<unsigned>(a.p.max_rows) * a.cluster, static_cast<unsigned>(a.p.heads), static_cast<unsigned>(a.p.n_seqs));
  if (a.padded == 64) return launch_clusters(a.cluster, choose_kernel<64>, g, kChooseThreads, choose_smem<64>(a.head_tiles, pages), st, a);
  return launch_clusters(a.cluster, choose_kernel<128>, g, kChooseThreads, choose_smem<128>(a.head_tiles, pages), st, a);
}

}  // namespace ipv
