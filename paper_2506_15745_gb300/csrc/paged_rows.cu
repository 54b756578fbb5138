// Rows into and out of a paged cache: a scatter of new rows to their pages,
// quantising them in 8 or 4 bits on the way, and the gather that reads them
// back. HBM-bound: every element is read once and written once. A team of
// lanes takes a K row and the matching V row: 4 lanes when writing, so that a
// group's minimum and maximum are two shuffles away and what a group costs beside
// its values is shared by 16 of them, 8 lanes when reading.
//
// Measured, 6272 rows of 112 heads of 128 channels, K and V, 4 bits: read 69 us (6.7
// TB/s); write 118 us for 68 us of bytes: no unit is busy more than 61% (issue, at about
// 16 instructions per value; ALU 53%, DRAM 35%), 3 blocks per SM (79 registers) wait for
// their loads and shuffles.
#include "paged_codes.cuh"

namespace ipv {
namespace {

constexpr int kBlock = 256;
constexpr int kTeam = 4;              // lanes that write a row, two chunks of a group each
constexpr int kTeams = kBlock / 8;    // rows that a block reads

// A new row of a head: where it lies in the packed rows, and which of its
// sequence's rows it is.
struct Item {
  int64_t packed;  // element of its first channel in the packed rows
  int j, h;
  bool in;         // there is such a row
};

__device__ __forceinline__ Item item_of(const RowsArgs& a, const Seq& s, int item, int items) {
  Item it;
  it.in = item < items;
  const int i = it.in ? item : 0, r = a.by_heads(i);
  it.h = i - r * a.p.heads;
  it.packed = (s.row0 + static_cast<int64_t>(r)) * a.row + it.h * a.head;
  it.j = s.len - s.n + r;
  return it;
}

// Its row of the pool (head included), -1: none.
__device__ __forceinline__ int64_t row_of(const RowsArgs& a, int b, const Item& it) {
  if (!it.in || it.j < 0) return -1;
  const int64_t row = pool_row(a.p, b, it.j);
  return row < 0 ? row : row + it.h * a.p.head_stride;
}

// A team takes a row of K and of V, both groups of them.
constexpr int kGroups = 2;

template <int FMT>
__global__ void __launch_bounds__(kBlock) write_kernel(RowsArgs a) {
  pdl_trigger();
  pdl_wait();
  const int b = blockIdx.y;
  const Seq s = sequence(a.p, b);
  const int items = s.n * a.p.heads;
  if (static_cast<int>(blockIdx.x) * (kBlock / kTeam) >= items) return;
  const int c = threadIdx.x & (kTeam - 1);
  const Item it = item_of(a, s, blockIdx.x * (kBlock / kTeam) + threadIdx.x / kTeam, items);
  uint4 xk[kGroups][2], xv[kGroups][2];
#pragma unroll
  for (int g = 0; g < kGroups; ++g)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int ch = g * kGroup + (c + kTeam * i) * 8;
      xk[g][i] = xv[g][i] = make_uint4(0, 0, 0, 0);
      if (it.in && ch < a.p.dim) {  // on their way while the page is looked up
        xk[g][i] = ld_once(a.k_new + it.packed + ch);
        xv[g][i] = ld_once(a.v_new + it.packed + ch);
      }
    }
  const int64_t row = row_of(a, b, it), at = row * a.p.row_bytes, par = row * a.p.groups;
#pragma unroll
  for (int g = 0; g < kGroups; ++g) {
    if (FMT == kBf16) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int ch = g * kGroup + (c + kTeam * i) * 8;
        if (row >= 0 && ch < a.p.dim) {
          *reinterpret_cast<uint4*>(a.p.k + at + 2 * ch) = xk[g][i];
          *reinterpret_cast<uint4*>(a.p.v + at + 2 * ch) = xv[g][i];
        }
      }
    } else if (g < a.p.groups) {  // whole warps
      uint32_t wk[4], wv[4];
      const uint32_t pk = quantise<FMT, 2>(xk[g], wk), pv = quantise<FMT, 2>(xv[g], wv);
      if (row >= 0) {
        uint32_t* kd = reinterpret_cast<uint32_t*>(a.p.k + at) + g * (FMT == kU8 ? kGroup / 4 : kGroup / 8);
        uint32_t* vd = reinterpret_cast<uint32_t*>(a.p.v + at) + g * (FMT == kU8 ? kGroup / 4 : kGroup / 8);
        if (FMT == kU8) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int word = 2 * (c + kTeam * (i >> 1)) + (i & 1);
            kd[place_u8(word)] = wk[i];
            vd[place_u8(word)] = wv[i];
          }
        } else {  // words c and c + 4 lie side by side
          *reinterpret_cast<uint2*>(kd + place_u4(c)) = make_uint2(wk[0], wk[1]);
          *reinterpret_cast<uint2*>(vd + place_u4(c)) = make_uint2(wv[0], wv[1]);
        }
        if (c == 0) a.p.k_par[par + g] = pk;
        if (c == 1) a.p.v_par[par + g] = pv;
      }
    }
  }
}

template <int FMT>
__global__ void __launch_bounds__(kBlock) read_kernel(RowsArgs a) {
  pdl_trigger();
  pdl_wait();
  const int b = blockIdx.y;
  const Seq s = sequence(a.p, b);
  const int items = s.n * a.p.heads;
  if (static_cast<int>(blockIdx.x) * kTeams >= items) return;
  const int c = threadIdx.x & 7;
  const Item it = item_of(a, s, blockIdx.x * kTeams + (threadIdx.x >> 3), items);
  const int64_t row = row_of(a, b, it), at = row * a.p.row_bytes, par = row * a.p.groups;
  uint4 xk[kGroups], xv[kGroups];  // bf16: the elements; codes: two words and the pair
#pragma unroll
  for (int g = 0; g < kGroups; ++g) {
    xk[g] = xv[g] = make_uint4(0, 0, 0, 0);
    if (row < 0 || g * kGroup + c * 8 >= a.p.dim) continue;
    if (FMT == kBf16) {
      xk[g] = ld_once(a.p.k + at + g * (2 * kGroup) + c * 16);
      xv[g] = ld_once(a.p.v + at + g * (2 * kGroup) + c * 16);
    } else {
      const uint32_t* kd = reinterpret_cast<const uint32_t*>(a.p.k + at) + g * (FMT == kU8 ? kGroup / 4 : kGroup / 8);
      const uint32_t* vd = reinterpret_cast<const uint32_t*>(a.p.v + at) + g * (FMT == kU8 ? kGroup / 4 : kGroup / 8);
      if (FMT == kU8) {
        xk[g].x = kd[place_u8(2 * c)], xk[g].y = kd[place_u8(2 * c + 1)];
        xv[g].x = vd[place_u8(2 * c)], xv[g].y = vd[place_u8(2 * c + 1)];
      } else {
        xk[g].x = kd[place_u4(c)];
        xv[g].x = vd[place_u4(c)];
      }
      xk[g].z = a.p.k_par[par + g];
      xv[g].z = a.p.v_par[par + g];
    }
  }
  if (!it.in) return;
#pragma unroll
  for (int g = 0; g < kGroups; ++g) {
    if (g * kGroup + c * 8 >= a.p.dim) continue;
    if (FMT != kBf16) {
      const uint32_t wk[2] = {xk[g].x, xk[g].y}, wv[2] = {xv[g].x, xv[g].y};
      xk[g] = expand<FMT, false>(wk, xk[g].z);
      xv[g] = expand<FMT, false>(wv, xv[g].z);
    }
    *reinterpret_cast<uint4*>(a.k_out + it.packed + g * kGroup + c * 8) = xk[g];
    *reinterpret_cast<uint4*>(a.v_out + it.packed + g * kGroup + c * 8) = xv[g];
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
  const int skip = a.sinks > 0 ? min(lo / a.step, (a.sinks - 1) / a.step + 1) * a.step : 0;  // sinks may be near 2^31
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

dim3 grid_of(const RowsArgs& a, int rows) {  // rows of a block
  const int64_t items = static_cast<int64_t>(a.p.max_rows) * a.p.heads;  // < 2^31, checked
  return dim3(static_cast<unsigned>((items + rows - 1) / rows), static_cast<unsigned>(a.p.n_seqs));
}

}  // namespace

cudaError_t launch_pages_write(const RowsArgs& a, cudaStream_t st) {
  switch (a.p.fmt) {
    case kBf16: return launch_next(write_kernel<kBf16>, grid_of(a, kBlock / kTeam), kBlock, 0, st, a);
    case kU8: return launch_next(write_kernel<kU8>, grid_of(a, kBlock / kTeam), kBlock, 0, st, a);
    default: return launch_next(write_kernel<kU4>, grid_of(a, kBlock / kTeam), kBlock, 0, st, a);
  }
}

cudaError_t launch_pages_read(const RowsArgs& a, cudaStream_t st) {
  switch (a.p.fmt) {
    case kBf16: return launch_next(read_kernel<kBf16>, grid_of(a, kTeams), kBlock, 0, st, a);
    case kU8: return launch_next(read_kernel<kU8>, grid_of(a, kTeams), kBlock, 0, st, a);
    default: return launch_next(read_kernel<kU4>, grid_of(a, kTeams), kBlock, 0, st, a);
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
