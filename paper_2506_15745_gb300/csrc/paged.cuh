// Internal declarations of the paged cache (paged.cu: C ABI; paged_rows.cu:
// write and read-back; rotate.cu: norms and rotation on the way in; bounds.cu:
// bounds of pages and the choice by them; move.cu: pages and rows moved;
// attend_rows.cu: attention of a few query rows, over all pages or chosen ones;
// attend_tiles.cu: of many).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "ipv_common.cuh"

namespace ipv {

// Division of 0 <= x < 2^31 by a fixed 1 <= d < 2^31 as a multiplication:
// x / d = x * m >> 31 + s with s = ceil(log2 d), m = ceil(2^(31 + s) / d); m is
// too large by less than 2^s / 2^(31 + s) of itself, which x cannot make a unit.
struct Divide {
  uint32_t m = 0;
  int s = 0, d = 1;
  Divide() = default;
  explicit Divide(int by) : d(by) {
    while ((int64_t{1} << s) < by) ++s;
    m = static_cast<uint32_t>(((uint64_t{1} << (31 + s)) + by - 1) / by);
  }
  __device__ __forceinline__ int operator()(int x) const {
    return static_cast<int>((static_cast<uint64_t>(static_cast<uint32_t>(x)) * m) >> (31 + s));
  }
};

enum : int { kBf16 = 0, kU8 = 1, kU4 = 2 };  // ipv_pages_format

constexpr int kGroup = 64;            // channels that share a step and a minimum
constexpr float kLargest = 32768.0f;  // a group with a larger magnitude is marked

// A pool and the sequences in it, as the kernels take them.
struct Pages {
  int fmt;
  int heads, dim;
  int page_size;
  int page_shift;      // log2(page_size); 31 with one page per sequence
  int n_pages, max_pages;
  int64_t page_stride, head_stride, row_stride;  // rows
  int row_bytes;       // of codes or elements
  int groups;          // (dim + 63) / 64
  char* k;
  char* v;
  uint32_t* k_par;     // pairs of fp16 (step, minimum)
  uint32_t* v_par;
  const int32_t* table;
  int64_t table_stride;
  const int32_t* row_start;
  const int32_t* kv_len;
  int n_seqs;
  int64_t total_rows;
  int max_rows, max_kv;  // max_kv already cut to max_pages * page_size
};

// New rows and length of a sequence, made to fit.
struct Seq {
  int row0, n, len;
};

__device__ __forceinline__ Seq sequence(const Pages& p, int b) {
  Seq s;
  const int r0 = p.row_start[b], r1 = p.row_start[b + 1];
  const int len = p.kv_len[b];
  s.row0 = r0;
  s.len = min(max(len, 0), p.max_kv);
  s.n = (r0 < 0 || r1 < r0 || r1 > p.total_rows) ? 0 : min(r1 - r0, p.max_rows);
  return s;
}

// Row number in the pool of row j >= 0 of sequence b (head's offset not
// included), or -1 if its page is not one of the pool's.
__device__ __forceinline__ int64_t pool_row(const Pages& p, int b, int j) {
  const int i = j >> p.page_shift;
  const int g = p.table ? p.table[b * p.table_stride + i] : b;
  if (static_cast<unsigned>(g) >= static_cast<unsigned>(p.n_pages)) return -1;
  return g * p.page_stride + (p.page_shift == 31 ? j : j & (p.page_size - 1)) * p.row_stride;
}

// Every kernel of the paged cache is launched to overlap its predecessor's end: it
// waits with pdl_wait() before it reads or writes anything, and lets its own
// successor be launched with pdl_trigger().
template <typename... Params, typename... Args>
cudaError_t launch_clusters(int cluster, void (*kernel)(Params...), dim3 grid, unsigned block, size_t smem, cudaStream_t st,
                            const Args&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(block);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = static_cast<unsigned>(cluster);
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}
template <typename... Params, typename... Args>
cudaError_t launch_next(void (*kernel)(Params...), dim3 grid, unsigned block, size_t smem, cudaStream_t st, const Args&... args) {
  return launch_clusters(1, kernel, grid, block, smem, st, args...);
}

// ------------------------------------------------------------------ attention
constexpr int kInTurn = -1;  // AttendArgs::unit
struct AttendArgs {
  Pages p;
  const uint16_t* q;
  uint16_t* out;
  float* lse;
  int64_t q_row, q_head, out_row, out_head;  // strides in elements
  int q_heads, share;   // query heads; query heads per KV head
  Divide by_share, by_tiles;
  int tiles;            // row tiles of max_rows
  float scale_log2;     // scale * log2(e)
  int causal, window, sinks;
  // Fewest units (steps and runs' costs) of a block's share; 0: `cluster` blocks (1, or 8 as one cluster,
  // which joins their parts by itself) take one KV head of one row tile; kInTurn (chosen pages): a block takes
  // tiles whole, every gridDim.x-th one.
  int unit, cluster;
  int tile;  // query rows of a row tile
  // Chosen pages: a row tile holds one new row's query heads (or `tile` of them), `per_row` tiles a new row; entry
  // e of chosen[row][KV head] is a page of the row's sequence. Keys count through the row's list: n_chosen pages
  // at most.
  const int32_t* chosen;
  int64_t chosen_row, chosen_head;
  int n_chosen;
  Divide by_per_row;
  int per_row;
  // Partial results, for each block's first and last run: unnormalised sums
  // (rows kernel: [blocks][2][tile][dim], tiled kernel: [blocks][2][dim / 4][tile][4]),
  // (running maximum, sum) [blocks][2][tile], and a record [blocks][2] (part_record).
  float* part_o;
  float2* part_ml;
  int4* part_rec;
};

// The steps of keys that query rows of tokens tok0..tok1 can see: steps
// 0..sink_steps-1 of the sequence, then those from first on, `steps` in all.
struct KeyRange {
  int sink_steps, first, steps;
  int hi_min, hi_max;  // keys j < hi of the first and of the last token
  int lo_max;          // the last token's window starts here
  template <int STEP>
  __device__ __forceinline__ int key0(int i) const {
    return (i < sink_steps ? i : i - sink_steps + first) * STEP;
  }
};

__device__ __forceinline__ int token_hi(const AttendArgs& a, const Seq& s, int tok) {
  return a.causal ? max(0, s.len - s.n + tok + 1) : s.len;
}

// Pages of a sequence that hold rows which token `tok` sees.
__device__ __forceinline__ int pages_seen(const AttendArgs& a, const Seq& s, int tok) {
  const int hi = token_hi(a, s, tok);
  return hi > 0 ? ((hi - 1) >> a.p.page_shift) + 1 : 0;
}

// The steps over the pages that token `tok` has chosen: keys count through its list. A row that sees one page ends in it at
// itself, however long the page is (a cache without a table is one page). At most 2^30 keys: max_kv is checked to be no more,
// and several pages are powers of two below it.
template <int STEP>
__device__ __forceinline__ KeyRange chosen_range(const AttendArgs& a, const Seq& s, int tok) {
  KeyRange r = {};
  const int pages = pages_seen(a, s, tok);
  r.hi_min = r.hi_max = pages > 1 ? min(a.n_chosen, pages) * a.p.page_size : token_hi(a, s, tok);
  r.steps = r.hi_max > 0 ? (r.hi_max - 1) / STEP + 1 : 0;
  return r;
}

template <int STEP>
__device__ __forceinline__ KeyRange key_range(const AttendArgs& a, const Seq& s, int tok0, int tok1) {
  KeyRange r;
  r.hi_min = token_hi(a, s, tok0);
  r.hi_max = token_hi(a, s, tok1);
  const int lo = a.window ? max(0, r.hi_min - a.window) : 0;
  r.lo_max = a.window ? max(0, r.hi_max - a.window) : 0;
  r.first = lo / STEP;
  // (x - 1) / STEP + 1 rather than (x + STEP - 1) / STEP: x may be near 2^31
  r.sink_steps = a.sinks > 0 ? min(r.first, (a.sinks - 1) / STEP + 1) : 0;
  const int end = r.hi_max > 0 ? (r.hi_max - 1) / STEP + 1 : 0;
  r.steps = r.sink_steps + max(0, end - r.first);
  return r;
}

// ------------------------------------------------------------------ launches
struct RowsArgs {
  Pages p;
  const uint16_t* k_new;
  const uint16_t* v_new;
  uint16_t* k_out;
  uint16_t* v_out;
  int64_t row, head;  // strides of the packed rows, elements
  Divide by_heads;
};
cudaError_t launch_pages_write(const RowsArgs& a, cudaStream_t st);
cudaError_t launch_pages_read(const RowsArgs& a, cudaStream_t st);

struct RotateArgs {
  Pages p;
  const uint16_t* q;
  const uint16_t* k_new;
  const uint16_t* v_new;
  uint16_t* q_out;
  int64_t q_row, q_head, out_row, out_head, row, head;  // strides in elements; the last two of k_new and v_new
  int q_heads;
  const float* turns;        // [n_positions][rot]: cosines, sines
  int64_t n_positions;
  int rot;
  bool neighbours;           // pairs (2i, 2i + 1)
  int ends[3];               // where the first axes' frequencies end
  const int32_t* positions;  // [axes][positions_stride]
  int64_t positions_stride;
  const uint16_t* q_weight;  // norms' weights, or NULL
  const uint16_t* k_weight;
  float eps, by_dim;
  int row_warps_shift;       // 1, 2 or 4 warps for a row: 0, 1 or 2
};
cudaError_t launch_rotate(const RotateArgs& a, cudaStream_t st);

// Whole pages of one pool: `to[i]` becomes a copy of `from[i]`.
struct CopyArgs {
  Pages p;                        // the pool alone
  const int32_t* from;
  const int32_t* to;
  int chunks, row_chunks, parts;  // 16-byte chunks of K in a page and in a row; blocks of a page
  Divide by_row, by_page, by_parts;
};
int pages_copy_part();            // chunks that a block copies
cudaError_t launch_pages_copy(const CopyArgs& a, int64_t n, cudaStream_t st);

// New row i of sequence b and head h in p becomes row kept[b][h][i] of sequence b in src.
struct MoveArgs {
  Pages p, src;
  const int32_t* kept;            // NULL: row i
  int64_t kept_seq, kept_head;
  int row_chunks;
};
cudaError_t launch_pages_gather(const MoveArgs& a, cudaStream_t st);

// Bounds of pages: codes [n_pages][heads][2][padded] (lower, upper), steps [n_pages][heads].
struct BoundsArgs {
  Pages p;
  char* codes;
  float* steps;
  int padded;
};
cudaError_t launch_bounds(const BoundsArgs& a, int pages, cudaStream_t st);  // pages that a sequence's new rows lie in, at most

struct ChooseArgs {
  Pages p;                        // the batch and the pool's shape; no rows are read
  const char* codes;
  const float* steps;
  int padded;
  const uint16_t* q;
  int64_t q_row, q_head;
  int share, head_tiles;          // query heads per KV head, in tiles of 8
  int32_t* out;
  int64_t out_row, out_head;
  int n, first, recent;
  int max_pages;                  // that a sequence has
  int cluster;                    // blocks that score the pages of one row and KV head
};
constexpr int kChooseThreads = 256;
constexpr int kChooseSmem = 227 * 1024;
cudaError_t choose_prepare();     // once per device
cudaError_t launch_choose(const ChooseArgs& a, int pages, cudaStream_t st);

// Every row that the new rows of a sequence may read, widened from codes to
// fp16 [n_seqs][heads][max_kv][dim]; rows that no step of `step` keys reads
// are left out.
struct ExpandArgs {
  Pages p;
  uint16_t* k_out;
  uint16_t* v_out;
  int causal, window, sinks, step;
};
cudaError_t launch_pages_expand(const ExpandArgs& a, cudaStream_t st);

int attend_rows_tile(int rows);               // query rows of a row tile
int attend_rows_resident(int fmt, int dim, int tile);  // blocks per SM, after attend_rows_prepare
constexpr int kRowsStep = 32;                 // keys of a step
constexpr int kRowsWarps = 4;
constexpr int kRowsCluster = 8;               // blocks of a cluster
cudaError_t attend_rows_prepare();            // once per device
cudaError_t launch_attend_rows(const AttendArgs& a, int blocks, cudaStream_t st);
int attend_chosen_resident(int fmt, int dim, int tile);  // the same for chosen pages
cudaError_t attend_chosen_prepare();
cudaError_t launch_attend_chosen(const AttendArgs& a, int blocks, cudaStream_t st);

// Many query rows (attend_tiles.cu): the pool's rows are 16-bit elements.
constexpr int kTilesRows = 256;  // query rows of a tile of work
constexpr int kTilesStep = 128;  // keys of a step
struct alignas(128) TileMaps {    // the pool as TMA sees it
  unsigned char k[128], v[128];
  int box_rows;                  // rows of a copy
};
cudaError_t attend_tiles_prepare();  // once per device
bool attend_tiles_maps(const AttendArgs& a, bool bf16, TileMaps* maps);
cudaError_t launch_attend_tiles(const AttendArgs& a, bool bf16, const TileMaps& maps, int blocks, int64_t limit_ns, cudaStream_t st);
cudaError_t attend_tiles_error(unsigned* bits);

}  // namespace ipv
