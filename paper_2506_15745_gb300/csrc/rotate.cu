// New rows on their way into the cache: queries and keys normalised per head and
// rotated by their positions in one pass, queries to the packed result, keys and
// values to their pages (quantised as paged_rows.cu does).
//
// A row is read once and written once. 8 lanes take a head of a row, lane c the
// 16-byte chunks c and c + 8, so that with all of 128 channels rotated in halves a
// lane has both ends of its pairs; elsewhere the partners come by shuffles. 1, 2 or 4
// warps take a row: their lanes fetch its cosines and sines once and use them for
// all the heads that they take, the next four heads on their way meanwhile. 16 frames
// (59 MB, 9 us at the copy rate) take 13.6 us, 16.0 into 8 and 4 bits; issue slots (66%), at about 320
// instructions per four heads, and the look-ups at a row's start (position, then angles;
// sequence, then page). The bf16 instance for all of 128 channels in halves has 80 registers and no spills with 6 blocks per SM,
// at 64 registers it spills (16.3 us); those into codes spill 52 bytes at 80. Rows of 64 channels have one chunk
// for a lane (784 rows of 32 + 8 heads 4.8 us; with an empty second chunk 7.1).
#include "paged_codes.cuh"

namespace ipv {
namespace {

constexpr int kBlock = 128;
constexpr int kBlockWarps = kBlock / 32;

// Pairs of channels: (i, i + 64) of 128, (i, i + rot / 2) of the first rot, (2i, 2i + 1).
enum : int { kOwn = 0, kHalves = 1, kNeighbours = 2 };

struct Turn {
  float c[8], s[8];  // kNeighbours: 4 of each
};

// Cosines and sines from frequency f on, N of them, of one axis.
template <int N>
__device__ __forceinline__ void load_turn(const RotateArgs& a, int64_t row, int f, Turn& x) {
  int axis = 0;
#pragma unroll
  for (int i = 0; i < 3; ++i) axis += f >= a.ends[i];
  const int pos = a.positions[axis * a.positions_stride + row];
  const bool in = static_cast<unsigned>(pos) < static_cast<unsigned>(a.n_positions);
  const float4* p = reinterpret_cast<const float4*>(a.turns + static_cast<int64_t>(in ? pos : 0) * a.rot + f);
  const float bad = __uint_as_float(0x7FC00000u);  // a position that the table has not
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    const float4 c = in ? p[i] : make_float4(bad, bad, bad, bad), s = in ? p[a.rot / 8 + i] : make_float4(bad, bad, bad, bad);
    x.c[4 * i] = c.x, x.c[4 * i + 1] = c.y, x.c[4 * i + 2] = c.z, x.c[4 * i + 3] = c.w;
    x.s[4 * i] = s.x, x.s[4 * i + 1] = s.y, x.s[4 * i + 2] = s.z, x.s[4 * i + 3] = s.w;
  }
}

__device__ __forceinline__ void unpack(const uint4& x, float (&y)[8]) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) y[2 * i] = lo_f(w[i]), y[2 * i + 1] = hi_f(w[i]);
}
__device__ __forceinline__ uint4 pack(const float (&y)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(y[2 * i + 1]), "f"(y[2 * i]));
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// A head's row, chunk c and, where rows have more than 64 channels (G = 2), chunk c + 8 of it in x: normalised with
// w (NULL: not), rotated. For whole warps, of which some teams may have queries, some keys, and one kind no norm.
template <int PAIRS, int G>
__device__ __forceinline__ void rotate(const RotateArgs& a, uint4 (&x)[G], const uint16_t* w, const Turn (&turn)[G], int c) {
  float y[G][8];
#pragma unroll
  for (int g = 0; g < G; ++g) unpack(x[g], y[g]);
  auto two = [](float (&z)[8], int i) { return make_float2(z[2 * i], z[2 * i + 1]); };  // packed arithmetic, two channels at once
  auto put = [](float (&z)[8], int i, float2 v) { z[2 * i] = v.x, z[2 * i + 1] = v.y; };
  if (a.q_weight || a.k_weight) {
    float2 sums = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int i = 0; i < 4; ++i) sums = fma2(two(y[g], i), two(y[g], i), sums);
    float sum = sums.x + sums.y;
#pragma unroll
    for (int d = 1; d < 8; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    const float inv = rsqrtf(sum * a.by_dim + a.eps);
#pragma unroll
    for (int g = 0; g < G; ++g) {
      if (!w || 8 * (c + 8 * g) >= a.p.dim) continue;
      float v[8];
      unpack(*reinterpret_cast<const uint4*>(w + 8 * (c + 8 * g)), v);
#pragma unroll
      for (int i = 0; i < 4; ++i) put(y[g], i, __fmul2_rn(two(y[g], i), __fmul2_rn(two(v, i), make_float2(inv, inv))));
    }
  }
  if constexpr (PAIRS == kOwn) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float lo = y[0][i], hi = y[1][i];
      y[0][i] = lo * turn[0].c[i] - hi * turn[0].s[i];
      y[1][i] = hi * turn[0].c[i] + lo * turn[0].s[i];
    }
  } else if constexpr (PAIRS == kNeighbours) {
#pragma unroll
    for (int g = 0; g < G; ++g) {
      if (8 * (c + 8 * g) >= a.rot) continue;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float lo = y[g][2 * i], hi = y[g][2 * i + 1];
        y[g][2 * i] = lo * turn[g].c[i] - hi * turn[g].s[i];
        y[g][2 * i + 1] = hi * turn[g].c[i] + lo * turn[g].s[i];
      }
    }
  } else if (G == 1 || a.rot <= 64) {  // all in the first chunks
    const int half = a.rot / 16, other = c < half ? c + half : c - half;  // any lane for a chunk that is not rotated
    float z[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = __shfl_sync(0xffffffffu, y[0][i], other & 7, 8);
    if (c < 2 * half)
#pragma unroll
      for (int i = 0; i < 8; ++i) y[0][i] = y[0][i] * turn[0].c[i] + (c < half ? -z[i] : z[i]) * turn[0].s[i];
  } else if constexpr (G == 2) {
    const int half = a.rot / 16;  // in chunks
    float z[G][8];
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const int n = c + 8 * g, other = n < half ? n + half : n - half;  // any lane for a chunk that is not rotated
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float u = __shfl_sync(0xffffffffu, y[0][i], other & 7, 8), v = __shfl_sync(0xffffffffu, y[1][i], other & 7, 8);
        z[g][i] = other & 8 ? v : u;
      }
    }
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const int n = c + 8 * g;
      if (n >= 2 * half) continue;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        y[g][i] = n < half ? y[g][i] * turn[g].c[i] - z[g][i] * turn[g].s[i] : y[g][i] * turn[g].c[i] + z[g][i] * turn[g].s[i];
    }
  }
#pragma unroll
  for (int g = 0; g < G; ++g) x[g] = pack(y[g]);
}

// One chunk of each group of a row of K or V into the pool.
template <int FMT, int G>
__device__ __forceinline__ void store(const Pages& p, char* pool, uint32_t* par, int64_t row, const uint4 (&x)[G], int c) {
#pragma unroll
  for (int g = 0; g < G; ++g) {
    if (FMT == kBf16) {
      if (row >= 0 && 8 * (c + 8 * g) < p.dim) *reinterpret_cast<uint4*>(pool + row * p.row_bytes + 16 * (c + 8 * g)) = x[g];
    } else if (g < p.groups) {  // whole warps
      const uint4 one[1] = {x[g]};
      uint32_t w[2];
      const uint32_t pair = quantise<FMT, 1>(one, w);
      if (row < 0) continue;
      uint32_t* to = reinterpret_cast<uint32_t*>(pool + row * p.row_bytes) + g * (FMT == kU8 ? kGroup / 4 : kGroup / 8);
      if (FMT == kU8) {
        to[place_u8(2 * c)] = w[0];
        to[place_u8(2 * c + 1)] = w[1];
      } else {
        to[place_u4(c)] = w[0];
      }
      if (c == 0) par[row * p.groups + g] = pair;
    }
  }
}

// The sequence whose new rows a packed row lies among: the last that starts at or before it. For whole warps.
__device__ __forceinline__ int sequence_of(const Pages& p, int64_t row) {
  const int lane = threadIdx.x & 31;
  int first = 0, n = p.n_seqs;
  while (true) {
    const int step = (n + 31) / 32, b = first + lane * step;
    const int before = __popc(__ballot_sync(0xffffffffu, b < first + n && p.row_start[b] <= row));
    first += max(0, before - 1) * step;
    if (step == 1) return first;
    n = min(step, p.n_seqs - first);
  }
}

template <int FMT, int PAIRS, int G>
__global__ void __launch_bounds__(kBlock, PAIRS == kOwn || G == 1 ? 6 : 4) rotate_kernel(RotateArgs a) {
  pdl_trigger();
  pdl_wait();
  const int warp = threadIdx.x >> 5, shift = a.row_warps_shift, row_warps = 1 << shift;
  const int64_t row = blockIdx.x * static_cast<int64_t>(kBlockWarps >> shift) + (warp >> shift);
  const int c = threadIdx.x & 7, items = a.q_heads + a.p.heads;
  const int first = (warp & (row_warps - 1)) * 4, mine = (threadIdx.x & 31) >> 3;  // a warp's items, the team's among them
  if (first >= items || row >= a.p.total_rows) return;
  auto load = [&](const uint16_t* from, uint4 (&x)[G], bool in) {
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const int ch = 8 * (c + 8 * g);
      x[g] = make_uint4(0, 0, 0, 0);
      if (in && ch < a.p.dim) x[g] = ld_once(from + ch);
    }
  };
  auto load_item = [&](int base, uint4 (&x)[G], uint4 (&v)[G]) {
    const int item = base + mine, h = item - a.q_heads;
    load(h < 0 ? a.q + row * a.q_row + item * a.q_head : a.k_new + row * a.row + h * a.head, x, item < items);
    if (base + 4 > a.q_heads) load(a.v_new + row * a.row + h * a.head, v, h >= 0 && item < items);
  };
  uint4 x[G], v[G] = {};
  load_item(first, x, v);  // on their way while positions, turns, sequence and page are looked up
  Turn turn[G];
  if (PAIRS == kOwn) {
    load_turn<8>(a, row, 8 * c, turn[0]);
  } else {
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const int n = c + 8 * g, half = a.rot / 16;
      if (n >= 2 * half) continue;
      if (PAIRS == kNeighbours)
        load_turn<4>(a, row, 4 * n, turn[g]);
      else
        load_turn<8>(a, row, 8 * (n < half ? n : n - half), turn[g]);
    }
  }
  const int b = sequence_of(a.p, row);
  const Seq s = sequence(a.p, b);
  if (row < s.row0 || row >= s.row0 + static_cast<int64_t>(s.n)) return;  // the same for the warp
  const int j = s.len - s.n + static_cast<int>(row - s.row0);
  for (int base = first; base < items; base += 4 * row_warps) {  // the same for a whole warp
    const int item = base + mine, h = item - a.q_heads;
    const bool in = item < items, q = in && h < 0;
    uint4 x_next[G] = {}, v_next[G] = {};
    if (base + 4 * row_warps < items) load_item(base + 4 * row_warps, x_next, v_next);
    int64_t to = -1;
    if (base + 4 > a.q_heads) {
      if (in && !q && j >= 0) to = pool_row(a.p, b, j);
      if (to >= 0) to += h * a.p.head_stride;
      store<FMT, G>(a.p, a.p.v, a.p.v_par, to, v, c);
    }
    rotate<PAIRS, G>(a, x, q ? a.q_weight : a.k_weight, turn, c);
    if (q) {
#pragma unroll
      for (int g = 0; g < G; ++g)
        if (8 * (c + 8 * g) < a.p.dim) *reinterpret_cast<uint4*>(a.q_out + row * a.out_row + item * a.out_head + 8 * (c + 8 * g)) = x[g];
    }
    if (base + 4 > a.q_heads) store<FMT, G>(a.p, a.p.k, a.p.k_par, to, x, c);
#pragma unroll
    for (int g = 0; g < G; ++g) x[g] = x_next[g], v[g] = v_next[g];
  }
}

template <int FMT>
cudaError_t launch(const RotateArgs& a, cudaStream_t st) {
  const int rows = kBlockWarps >> a.row_warps_shift;
  const dim3 g(static_cast<unsigned>((a.p.total_rows + rows - 1) / rows));
  if (a.p.dim <= 64)
    return a.neighbours ? launch_next(rotate_kernel<FMT, kNeighbours, 1>, g, kBlock, 0, st, a)
                        : launch_next(rotate_kernel<FMT, kHalves, 1>, g, kBlock, 0, st, a);
  if (a.neighbours) return launch_next(rotate_kernel<FMT, kNeighbours, 2>, g, kBlock, 0, st, a);
  if (a.rot == 128) return launch_next(rotate_kernel<FMT, kOwn, 2>, g, kBlock, 0, st, a);
  return launch_next(rotate_kernel<FMT, kHalves, 2>, g, kBlock, 0, st, a);
}

}  // namespace

cudaError_t launch_rotate(const RotateArgs& a, cudaStream_t st) {
  switch (a.p.fmt) {
    case kBf16: return launch<kBf16>(a, st);
    case kU8: return launch<kU8>(a, st);
    default: return launch<kU4>(a, st);
  }
}

}  // namespace ipv
