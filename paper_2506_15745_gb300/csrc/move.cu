// Rows from pages to pages, as they are: whole pages copied (a sequence forked),
// and rows that each head keeps gathered into other pages (a sequence compacted).
// HBM-bound: every byte is read once and written once, codes with their pairs of
// step and minimum beside them.
#include "paged_codes.cuh"

namespace ipv {
namespace {

constexpr int kBlock = 256;
constexpr int kAtOnce = 4;                     // 16-byte chunks of K, and of V, that a thread has on their way
constexpr int kPart = kBlock * kAtOnce;        // chunks of K that a block copies

// A block copies a part of one page: chunks part * kPart.. of its heads' rows, 8 loads of a thread on their way. 8 pages of
// 4 heads (1 MB) are a launch: 2.2 us in a graph. 1024 of them (268 MB in all) 42 us, 6.4 TB/s.
__global__ void __launch_bounds__(kBlock) copy_kernel(CopyArgs a) {
  pdl_trigger();
  pdl_wait();
  const int pair = a.by_parts(blockIdx.x), part = blockIdx.x - pair * a.parts;
  const int from = a.from[pair], to = a.to[pair];
  if (static_cast<unsigned>(from) >= static_cast<unsigned>(a.p.n_pages) || static_cast<unsigned>(to) >= static_cast<unsigned>(a.p.n_pages)) return;
  const int64_t src = from * a.p.page_stride, dst = to * a.p.page_stride;
  uint4 k[kAtOnce], v[kAtOnce];
  uint2 par[kAtOnce];
  int64_t row[kAtOnce];
  int c[kAtOnce];
#pragma unroll
  for (int i = 0; i < kAtOnce; ++i) {
    const int chunk = part * kPart + i * kBlock + threadIdx.x;
    row[i] = -1;
    if (chunk >= a.chunks) continue;
    const int r = a.by_row(chunk), h = a.by_page(r);
    c[i] = chunk - r * a.row_chunks;
    row[i] = h * a.p.head_stride + (r - h * a.p.page_size) * a.p.row_stride;
    const int64_t at = (src + row[i]) * a.p.row_bytes + c[i] * 16;
    k[i] = ld_once(a.p.k + at);
    v[i] = ld_once(a.p.v + at);
    if (a.p.fmt != kBf16 && c[i] < 2) {  // chunk 0 has K's pairs, chunk 1 V's
      const uint32_t* p = (c[i] == 0 ? a.p.k_par : a.p.v_par) + (src + row[i]) * a.p.groups;
      par[i] = a.p.groups == 2 ? *reinterpret_cast<const uint2*>(p) : make_uint2(*p, 0u);
    }
  }
#pragma unroll
  for (int i = 0; i < kAtOnce; ++i) {
    if (row[i] < 0) continue;
    const int64_t at = (dst + row[i]) * a.p.row_bytes + c[i] * 16;
    *reinterpret_cast<uint4*>(a.p.k + at) = k[i];
    *reinterpret_cast<uint4*>(a.p.v + at) = v[i];
    if (a.p.fmt != kBf16 && c[i] < 2) {
      uint32_t* p = (c[i] == 0 ? a.p.k_par : a.p.v_par) + (dst + row[i]) * a.p.groups;
      if (a.p.groups == 2)
        *reinterpret_cast<uint2*>(p) = par[i];
      else
        *p = par[i].x;
    }
  }
}

// A team of 8 lanes takes a row of K and of V of one head as one list of 16-byte
// chunks, T of them per lane, and 8 / T rows at once: 8 loads on their way in
// each lane whatever the format. Before that a thread for each row looks up (the kept index,
// then the pages) where it comes from and goes to. 112 heads of 9408 bf16 rows cut to 6272 (722 MB with the indices) 109.9 us,
// 6.6 TB/s, 97% of the copy rate; 8 streams' 4-bit rows cut to two thirds (199 MB) 44 us, 66%.
constexpr int kTeams = kBlock / 8;

template <int T>
__global__ void __launch_bounds__(kBlock) move_rows_kernel(MoveArgs a) {
  constexpr int kRows = 8 / T, kTile = kTeams * kRows;
  __shared__ longlong2 places[kTile];  // rows of the pools, head included; from: -1 reads as zero, to: -1 is dropped
  pdl_trigger();
  pdl_wait();
  const int b = blockIdx.z, h = blockIdx.y, first = blockIdx.x * kTile, lane = threadIdx.x & 7, team = threadIdx.x >> 3;
  const int i = first + static_cast<int>(threadIdx.x);
  const bool looks = threadIdx.x < kTile && i < a.p.max_rows;
  // The index does not wait for the lengths: a list has one for every row that a sequence may have.
  const int r = !looks ? -1 : a.kept ? a.kept[b * a.kept_seq + h * a.kept_head + i] : i;
  const Seq s = sequence(a.p, b);
  if (first >= s.n) return;
  const int held = min(max(a.src.kv_len[b], 0), a.src.max_kv), j = s.len - s.n + i;
  if (threadIdx.x < kTile) {
    longlong2 x = make_longlong2(-1, -1);
    if (i < s.n && j >= 0) {
      if (r >= 0 && r < held) x.x = pool_row(a.src, b, r);
      x.y = pool_row(a.p, b, j);
      if (x.x >= 0) x.x += h * a.src.head_stride;
      if (x.y >= 0) x.y += h * a.p.head_stride;
    }
    places[threadIdx.x] = x;
  }
  __syncthreads();
  const int chunks = a.row_chunks;
  uint4 x[kRows][T];
  uint2 par[kRows];
#pragma unroll
  for (int u = 0; u < kRows; ++u) {
    const int64_t row = places[team + u * kTeams].x;
#pragma unroll
    for (int t = 0; t < T; ++t) {
      const int c = lane + 8 * t;
      x[u][t] = make_uint4(0, 0, 0, 0);
      if (row >= 0 && c < 2 * chunks) x[u][t] = ld_once((c < chunks ? a.src.k + c * 16 : a.src.v + (c - chunks) * 16) + row * a.src.row_bytes);
    }
    par[u] = make_uint2(0, 0);
    if (a.p.fmt != kBf16 && row >= 0 && lane < 2) {
      const uint32_t* p = (lane == 0 ? a.src.k_par : a.src.v_par) + row * a.src.groups;
      par[u] = a.src.groups == 2 ? *reinterpret_cast<const uint2*>(p) : make_uint2(*p, 0u);
    }
  }
#pragma unroll
  for (int u = 0; u < kRows; ++u) {
    const int64_t row = places[team + u * kTeams].y;
    if (row < 0) continue;
#pragma unroll
    for (int t = 0; t < T; ++t) {
      const int c = lane + 8 * t;
      if (c < 2 * chunks) *reinterpret_cast<uint4*>((c < chunks ? a.p.k + c * 16 : a.p.v + (c - chunks) * 16) + row * a.p.row_bytes) = x[u][t];
    }
    if (a.p.fmt != kBf16 && lane < 2) {
      uint32_t* p = (lane == 0 ? a.p.k_par : a.p.v_par) + row * a.p.groups;
      if (a.p.groups == 2)
        *reinterpret_cast<uint2*>(p) = par[u];
      else
        *p = par[u].x;
    }
  }
}

template <int T>
cudaError_t launch_move(const MoveArgs& a, cudaStream_t st) {
  constexpr int kTile = kTeams * (8 / T);
  const dim3 g(static_cast<unsigned>((a.p.max_rows + kTile - 1) / kTile), static_cast<unsigned>(a.p.heads), static_cast<unsigned>(a.p.n_seqs));
  return launch_next(move_rows_kernel<T>, g, kBlock, 0, st, a);
}

}  // namespace

int pages_copy_part() { return kPart; }

cudaError_t launch_pages_copy(const CopyArgs& a, int64_t n, cudaStream_t st) {
  return launch_next(copy_kernel, dim3(static_cast<unsigned>(n * a.parts)), kBlock, 0, st, a);
}

cudaError_t launch_pages_gather(const MoveArgs& a, cudaStream_t st) {
  if (a.row_chunks <= 4) return launch_move<1>(a, st);
  if (a.row_chunks <= 8) return launch_move<2>(a, st);
  return launch_move<4>(a, st);
}

}  // namespace ipv
