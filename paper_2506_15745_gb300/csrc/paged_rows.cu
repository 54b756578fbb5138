// Rows into and out of a paged cache: a scatter of new rows to their pages,
// quantising them in 8 or 4 bits on the way, and the gather that reads them
// back. HBM-bound: every element is read once and written once. A team of 8
// lanes takes one group of 64 channels (16 bytes of bf16 per lane) of a K row
// and of the matching V row, so a group's minimum and maximum are three
// shuffles away and nothing but the row itself is ever held.
#include <cuda_fp16.h>

#include "paged.cuh"

namespace ipv {
namespace {

constexpr int kBlock = 256;
constexpr int kTeams = kBlock / 8;  // groups in flight per block and round

// Where a group's words lie (ipv.h, Codes): lane c of a team holds channels
// 8c..8c+7: word c at 4 bits, words 2c and 2c+1 at 8 bits.
__device__ __forceinline__ int place_u4(int c) { return 2 * (c & 3) + (c >> 2); }
__device__ __forceinline__ int place_u8(int word) { return 4 * (word & 3) + (word >> 2); }

__device__ __forceinline__ float lo_f(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// Quantises a lane's 8 channels with its team's other 56: codes in w (one word
// at 4 bits, two at 8), the group's (step, minimum) in the return value.
template <int FMT>
__device__ __forceinline__ uint32_t quantise(const uint4& x, uint32_t (&w)[2]) {
  constexpr float kLevels = FMT == kU8 ? 255.0f : 15.0f;
  const uint32_t xs[4] = {x.x, x.y, x.z, x.w};
  float f[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) f[2 * i] = lo_f(xs[i]), f[2 * i + 1] = hi_f(xs[i]);
  float lo = f[0], hi = f[0], far = 0.0f;
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    lo = fminf(lo, f[i]);
    hi = fmaxf(hi, f[i]);
    bad |= !(fabsf(f[i]) <= kLargest);  // NaN too
  }
#pragma unroll
  for (int d = 1; d < 8; d <<= 1) {
    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, d));
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, d));
  }
  const uint32_t any = __ballot_sync(0xffffffffu, bad) >> (threadIdx.x & 24);
  if (any & 0xffu) {
    w[0] = w[1] = 0;
    return 0x7FFF7FFFu;  // (NaN, NaN)
  }
  const __half hm = __float2half_rd(lo);
  const float m = __half2float(hm);
  const __half hs = __float2half_ru((hi - m) / kLevels);
  const float s = __half2float(hs);
  // u = rint((x - m) / s). The product with 1/s is within 3e-5 of the quotient,
  // so it rounds to the same integer unless it lies that near a half: only then
  // is the division done.
  const float inv = s > 0.0f ? __frcp_rn(s) : 0.0f;
  float u[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float q = (f[i] - m) * inv;
    u[i] = fminf(rintf(q), kLevels);
    far = fmaxf(far, fabsf(q - u[i]));
  }
  if (far > 0.4999f) {
#pragma unroll
    for (int i = 0; i < 8; ++i) u[i] = s > 0.0f ? fminf(rintf((f[i] - m) / s), kLevels) : 0.0f;
  }
  if (FMT == kU8) {
    // Two codes at a time: u0 + 256 u1 is exact in fp32.
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t a = static_cast<uint32_t>(fmaf(u[4 * i + 1], 256.0f, u[4 * i]));
      const uint32_t b = static_cast<uint32_t>(fmaf(u[4 * i + 3], 256.0f, u[4 * i + 2]));
      w[i] = a | (b << 16);
    }
  } else {
    uint32_t h[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
      h[i] = static_cast<uint32_t>(
          fmaf(fmaf(u[4 * i + 3], 16.0f, u[4 * i + 2]), 256.0f, fmaf(u[4 * i + 1], 16.0f, u[4 * i])));
    w[0] = h[0] | (h[1] << 16);
    w[1] = 0;
  }
  return __half_as_ushort(hs) | (static_cast<uint32_t>(__half_as_ushort(hm)) << 16);
}

// The inverse, rounded once to bf16, or to fp16.
template <int FMT, bool F16>
__device__ __forceinline__ uint4 expand(const uint32_t (&w)[2], uint32_t par) {
  const float s = __half2float(__ushort_as_half(static_cast<unsigned short>(par & 0xFFFFu)));
  const float m = __half2float(__ushort_as_half(static_cast<unsigned short>(par >> 16)));
  float f[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t u = FMT == kU8 ? (w[i >> 2] >> (8 * (i & 3))) & 255u : (w[0] >> (4 * i)) & 15u;
    f[i] = fmaf(static_cast<float>(u), s, m);
  }
  uint32_t o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (F16)
      asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(o[i]) : "f"(f[2 * i + 1]), "f"(f[2 * i]));
    else
      asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(o[i]) : "f"(f[2 * i + 1]), "f"(f[2 * i]));
  }
  return make_uint4(o[0], o[1], o[2], o[3]);
}

// One group of one new row: where it lies in the packed rows and in the pool.
struct Item {
  int64_t packed;  // element of the group's first channel in the packed rows
  int64_t row;     // row of the pool (head included), -1: none
  int g;           // group
  bool in;         // there is such a row
};

__device__ __forceinline__ Item item_of(const RowsArgs& a, const Seq& s, int b, unsigned item, unsigned items) {
  Item it;
  it.in = item < items;
  const unsigned i = it.in ? item : 0;
  const unsigned groups = a.p.groups, per_row = groups * a.p.heads;
  const unsigned r = i / per_row, hg = i - r * per_row;
  const unsigned h = groups == 2 ? hg >> 1 : hg;
  it.g = groups == 2 ? hg & 1 : 0;
  it.packed = (s.row0 + static_cast<int64_t>(r)) * a.row + h * a.head + it.g * kGroup;
  const int j = s.len - s.n + static_cast<int>(r);
  it.row = -1;
  if (it.in && j >= 0) {
    it.row = pool_row(a.p, b, j);
    if (it.row >= 0) it.row += h * a.p.head_stride;
  }
  return it;
}

template <int FMT, int U>
__global__ void __launch_bounds__(kBlock) write_kernel(RowsArgs a) {
  pdl_trigger();
  pdl_wait();
  const int b = blockIdx.y;
  const Seq s = sequence(a.p, b);
  const unsigned items = static_cast<unsigned>(s.n) * a.p.heads * a.p.groups;
  const unsigned base = blockIdx.x * (kTeams * U) + (threadIdx.x >> 3);
  if (blockIdx.x * (kTeams * U) >= items) return;
  const int c = threadIdx.x & 7;
  Item it[U];
  uint4 xk[U], xv[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    it[u] = item_of(a, s, b, base + u * kTeams, items);
    const bool ok = it[u].row >= 0 && it[u].g * kGroup + c * 8 < a.p.dim;
    xk[u] = xv[u] = make_uint4(0, 0, 0, 0);
    if (ok) {
      xk[u] = ld_stream(a.k_new + it[u].packed + c * 8);
      xv[u] = ld_stream(a.v_new + it[u].packed + c * 8);
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (FMT == kBf16) {
      if (it[u].row >= 0 && it[u].g * kGroup + c * 8 < a.p.dim) {
        const int64_t at = it[u].row * a.p.row_bytes + it[u].g * (2 * kGroup) + c * 16;
        *reinterpret_cast<uint4*>(a.p.k + at) = xk[u];
        *reinterpret_cast<uint4*>(a.p.v + at) = xv[u];
      }
    } else {
      uint32_t wk[2], wv[2];
      const uint32_t pk = quantise<FMT>(xk[u], wk), pv = quantise<FMT>(xv[u], wv);  // whole warps
      if (it[u].row >= 0) {
        const int64_t at = it[u].row * a.p.row_bytes + it[u].g * (FMT == kU8 ? kGroup : kGroup / 2);
        uint32_t* kd = reinterpret_cast<uint32_t*>(a.p.k + at);
        uint32_t* vd = reinterpret_cast<uint32_t*>(a.p.v + at);
        if (FMT == kU8) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            kd[place_u8(2 * c + i)] = wk[i];
            vd[place_u8(2 * c + i)] = wv[i];
          }
        } else {
          kd[place_u4(c)] = wk[0];
          vd[place_u4(c)] = wv[0];
        }
        const int64_t par = it[u].row * a.p.groups + it[u].g;
        if (c == 0) a.p.k_par[par] = pk;
        if (c == 1) a.p.v_par[par] = pv;
      }
    }
  }
}

template <int FMT, int U>
__global__ void __launch_bounds__(kBlock) read_kernel(RowsArgs a) {
  pdl_trigger();
  pdl_wait();
  const int b = blockIdx.y;
  const Seq s = sequence(a.p, b);
  const unsigned items = static_cast<unsigned>(s.n) * a.p.heads * a.p.groups;
  const unsigned base = blockIdx.x * (kTeams * U) + (threadIdx.x >> 3);
  if (blockIdx.x * (kTeams * U) >= items) return;
  const int c = threadIdx.x & 7;
  Item it[U];
  uint4 xk[U], xv[U];  // bf16: the elements; codes: two words and the pair
#pragma unroll
  for (int u = 0; u < U; ++u) {
    it[u] = item_of(a, s, b, base + u * kTeams, items);
    xk[u] = xv[u] = make_uint4(0, 0, 0, 0);
    if (it[u].row < 0) continue;
    if (FMT == kBf16) {
      if (it[u].g * kGroup + c * 8 < a.p.dim) {
        const int64_t at = it[u].row * a.p.row_bytes + it[u].g * (2 * kGroup) + c * 16;
        xk[u] = ld_stream(a.p.k + at);
        xv[u] = ld_stream(a.p.v + at);
      }
    } else {
      const int64_t at = it[u].row * a.p.row_bytes + it[u].g * (FMT == kU8 ? kGroup : kGroup / 2);
      const uint32_t* kd = reinterpret_cast<const uint32_t*>(a.p.k + at);
      const uint32_t* vd = reinterpret_cast<const uint32_t*>(a.p.v + at);
      if (FMT == kU8) {
        xk[u].x = kd[place_u8(2 * c)], xk[u].y = kd[place_u8(2 * c + 1)];
        xv[u].x = vd[place_u8(2 * c)], xv[u].y = vd[place_u8(2 * c + 1)];
      } else {
        xk[u].x = kd[place_u4(c)];
        xv[u].x = vd[place_u4(c)];
      }
      const int64_t par = it[u].row * a.p.groups + it[u].g;
      xk[u].z = a.p.k_par[par];
      xv[u].z = a.p.v_par[par];
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (!it[u].in || it[u].g * kGroup + c * 8 >= a.p.dim) continue;
    if (FMT != kBf16) {
      const uint32_t wk[2] = {xk[u].x, xk[u].y}, wv[2] = {xv[u].x, xv[u].y};
      xk[u] = expand<FMT, false>(wk, xk[u].z);
      xv[u] = expand<FMT, false>(wv, xv[u].z);
    }
    *reinterpret_cast<uint4*>(a.k_out + it[u].packed + c * 8) = xk[u];
    *reinterpret_cast<uint4*>(a.v_out + it[u].packed + c * 8) = xv[u];
  }
}

// Codes widened to fp16 for a kernel that takes 16-bit rows. A team's item is
// one group of one row of one head, rows innermost, so that the output is
// written in order.
template <int FMT, int U>
__global__ void __launch_bounds__(kBlock) expand_kernel(ExpandArgs a) {
  pdl_trigger();
  pdl_wait();
  const int b = blockIdx.z, h = blockIdx.y;
  const Seq s = sequence(a.p, b);
  if (s.n == 0) return;
  const unsigned groups = a.p.groups, items = static_cast<unsigned>(s.len) * groups;
  const unsigned base = blockIdx.x * (kTeams * U) + (threadIdx.x >> 3);
  // Rows skip..lo-1 lie between the sinks and the first new row's window.
  const int hi = a.causal ? max(0, s.len - s.n + 1) : s.len;
  const int lo = a.window ? max(0, hi - a.window) / a.step * a.step : 0;
  const int skip = a.sinks > 0 ? ((a.sinks - 1) / a.step + 1) * a.step : 0;
  const int c = threadIdx.x & 7;
  uint32_t wk[U][2], wv[U][2], pk[U], pv[U];
  int64_t out[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const unsigned item = base + u * kTeams;
    const int j = static_cast<int>(groups == 2 ? item >> 1 : item), g = groups == 2 ? item & 1 : 0;
    out[u] = -1;
    wk[u][0] = wk[u][1] = wv[u][0] = wv[u][1] = pk[u] = pv[u] = 0;
    if (item >= items || (j >= skip && j < lo)) continue;
    out[u] = ((static_cast<int64_t>(b) * a.p.heads + h) * a.p.max_kv + j) * a.p.dim + g * kGroup + c * 8;
    const int64_t r = pool_row(a.p, b, j);
    if (r < 0) continue;
    const int64_t row = r + h * a.p.head_stride;
    const int64_t at = row * a.p.row_bytes + g * (FMT == kU8 ? kGroup : kGroup / 2);
    const uint32_t* kd = reinterpret_cast<const uint32_t*>(a.p.k + at);
    const uint32_t* vd = reinterpret_cast<const uint32_t*>(a.p.v + at);
    if (FMT == kU8) {
      wk[u][0] = kd[place_u8(2 * c)], wk[u][1] = kd[place_u8(2 * c + 1)];
      wv[u][0] = vd[place_u8(2 * c)], wv[u][1] = vd[place_u8(2 * c + 1)];
    } else {
      wk[u][0] = kd[place_u4(c)];
      wv[u][0] = vd[place_u4(c)];
    }
    pk[u] = a.p.k_par[row * groups + g];
    pv[u] = a.p.v_par[row * groups + g];
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (out[u] < 0) continue;
    *reinterpret_cast<uint4*>(a.k_out + out[u]) = expand<FMT, true>(wk[u], pk[u]);
    *reinterpret_cast<uint4*>(a.v_out + out[u]) = expand<FMT, true>(wv[u], pv[u]);
  }
}

template <int U>
dim3 grid_of(const RowsArgs& a) {
  const int64_t items = static_cast<int64_t>(a.p.max_rows) * a.p.heads * a.p.groups;  // < 2^31, checked
  return dim3(static_cast<unsigned>((items + kTeams * U - 1) / (kTeams * U)), static_cast<unsigned>(a.p.n_seqs));
}

}  // namespace

cudaError_t launch_pages_write(const RowsArgs& a, cudaStream_t st) {
  const dim3 g = grid_of<2>(a);
  switch (a.p.fmt) {
    case kBf16: return launch_next(write_kernel<kBf16, 2>, g, kBlock, 0, st, a);
    case kU8: return launch_next(write_kernel<kU8, 2>, g, kBlock, 0, st, a);
    default: return launch_next(write_kernel<kU4, 2>, g, kBlock, 0, st, a);
  }
}

cudaError_t launch_pages_read(const RowsArgs& a, cudaStream_t st) {
  const dim3 g = grid_of<2>(a);
  switch (a.p.fmt) {
    case kBf16: return launch_next(read_kernel<kBf16, 2>, g, kBlock, 0, st, a);
    case kU8: return launch_next(read_kernel<kU8, 2>, g, kBlock, 0, st, a);
    default: return launch_next(read_kernel<kU4, 2>, g, kBlock, 0, st, a);
  }
}

cudaError_t launch_pages_expand(const ExpandArgs& a, cudaStream_t st) {
  constexpr int kU = 2;
  const int64_t items = static_cast<int64_t>(a.p.max_kv) * a.p.groups;
  const dim3 g(static_cast<unsigned>((items + kTeams * kU - 1) / (kTeams * kU)), static_cast<unsigned>(a.p.heads),
               static_cast<unsigned>(a.p.n_seqs));
  if (a.p.fmt == kU8)
    return launch_next(expand_kernel<kU8, kU>, g, kBlock, 0, st, a);
  return launch_next(expand_kernel<kU4, kU>, g, kBlock, 0, st, a);
}

}  // namespace ipv
