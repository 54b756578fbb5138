// How the attention kernels share out their work: blocks take equal runs of a
// list of all steps, in order; a tile whose keys several blocks share leaves a
// partial result in each, which a second kernel joins.
#pragma once

#include "paged.cuh"

namespace ipv {

// A tile of ROWS query rows of a sequence: pair number p = sequence * tiles + tile.
struct Tile {
  Seq seq;
  int b, row0, n_rows, steps;
  KeyRange kr;
  int number;  // of the tile in its sequence; CHOSEN only, elsewhere row0 / ROWS
};

// CHOSEN: a tile is ROWS of the query heads of one new row, over the row's chosen pages.
template <int ROWS, int STEP, bool CHOSEN = false>
__device__ __forceinline__ void set_tile(const AttendArgs& a, Tile& x, int b, int tile) {
  if constexpr (CHOSEN) {
    const int tok = a.by_per_row(tile), head0 = (tile - tok * a.per_row) * ROWS;
    x.number = tile;
    x.row0 = tok * a.share + head0;
    x.n_rows = tok < x.seq.n ? min(ROWS, a.share - head0) : 0;
    x.b = b;
    x.steps = 0;
    if (x.n_rows > 0) {
      x.kr = chosen_range<STEP>(a, x.seq, tok);
      x.steps = max(1, x.kr.steps);
    }
    return;
  }
  x.row0 = tile * ROWS;
  x.n_rows = min(ROWS, x.seq.n * a.share - x.row0);
  x.b = b;
  x.steps = 0;
  if (x.n_rows > 0) {
    x.kr = key_range<STEP>(a, x.seq, a.by_share(x.row0), a.by_share(x.row0 + x.n_rows - 1));
    x.steps = max(1, x.kr.steps);  // rows that see nothing have their results to write, too
  }
}
template <int ROWS, int STEP, bool CHOSEN = false>
__device__ __forceinline__ Tile tile_of(const AttendArgs& a, int tiles, int p) {
  Tile x;
  const int b = a.by_tiles(p);
  x.seq = sequence(a.p, b);
  set_tile<ROWS, STEP, CHOSEN>(a, x, b, p - b * tiles);
  return x;
}

// What the blocks share out: a tile's keys for one KV head weigh their steps and
// COST more, about what loading the queries, filling the pipeline and writing
// the results take. A block's share starts `at` units into KV head `head` of
// pair p and is `left` units long. Heads of a pair follow one another, then pairs.
struct Share {
  int p, head;
  int64_t at, left;
};

// 64-bit numbers that mostly fit 32 bits.
__device__ __forceinline__ int64_t divide(int64_t x, int64_t d) {
  if (static_cast<uint64_t>(x | d) >> 32 == 0) return static_cast<uint32_t>(x) / static_cast<uint32_t>(d);
  return x / d;
}

// Walks a share, a run of steps of one (pair, head) at a time. A boundary within
// the first COST units leaves all steps to the block behind it.
template <int ROWS, int STEP, int COST, bool CHOSEN = false>
struct Walk {
  Tile t;
  int head, s, n;  // steps s .. s + n - 1
  int64_t left;    // kInTurn: the number of the tile and head in its sequence, plus what the sequences before it have
  __device__ __forceinline__ void cut(int64_t at) {
    const int64_t weight = t.steps + COST, upto = min(weight, at + left);
    s = static_cast<int>(max(int64_t{0}, at - COST));
    n = static_cast<int>(max(int64_t{0}, upto - COST)) - s;
    left -= upto - at;
  }
  // kInTurn: the tile and head `left` places on from the first of sequence b, which is t.seq.
  __device__ __forceinline__ void place(const AttendArgs& a, int b) {
    const int64_t one = static_cast<int64_t>(t.seq.n) * a.per_row;
    head = static_cast<int>(divide(left, one));
    set_tile<ROWS, STEP, true>(a, t, b, static_cast<int>(left - head * one));
    s = 0;
    n = t.steps;
  }
  // The same where it may be a later sequence's, 32 sequences at a time. Heads of a sequence follow one
  // another, so that the blocks that run at the same time read pages of one head or two. For whole warps.
  __device__ __forceinline__ bool settle(const AttendArgs& a, int b) {
    const int lane = threadIdx.x & 31;
    for (; b < a.p.n_seqs; b += 32) {
      const int64_t mine = b + lane < a.p.n_seqs ? static_cast<int64_t>(sequence(a.p, b + lane).n) * a.per_row * a.p.heads : 0;
      int64_t upto = mine;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int64_t y = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= d) upto += y;
      }
      const uint32_t there = __ballot_sync(0xffffffffu, left < upto);
      if (there) {
        const int i = __ffs(there) - 1;
        left -= __shfl_sync(0xffffffffu, upto - mine, i);
        t.seq = sequence(a.p, b + i);
        place(a, b + i);
        return true;
      }
      left -= __shfl_sync(0xffffffffu, upto, 31);
    }
    return false;
  }
  __device__ __forceinline__ bool begin(const AttendArgs& a, int tiles, const Share& w) {
    if (CHOSEN && a.unit == kInTurn) {
      left = blockIdx.x;
      return settle(a, 0);
    }
    t = tile_of<ROWS, STEP, CHOSEN>(a, tiles, w.p);
    head = w.head;
    left = w.left;
    cut(w.at);
    return n > 0 || next(a, tiles);
  }
  __device__ __forceinline__ bool next(const AttendArgs& a, int tiles) {
    if (CHOSEN && a.unit == kInTurn) {
      left += gridDim.x;
      if (left >= static_cast<int64_t>(t.seq.n) * a.per_row * a.p.heads) return settle(a, t.b);
      place(a, t.b);
      return true;
    }
    if (left <= 0) return false;
    if (++head == a.p.heads) {
      head = 0;
      int tile = number(), b = t.b;
      do {
        if (++tile == tiles) {
          tile = 0;
          if (++b == a.p.n_seqs) return false;  // only if the lengths changed under the kernel
          t.seq = sequence(a.p, b);
        }
        set_tile<ROWS, STEP, CHOSEN>(a, t, b, tile);
      } while (t.steps == 0);
    }
    cut(0);
    return n > 0;
  }
  __device__ __forceinline__ bool starts() const { return s == 0; }
  __device__ __forceinline__ bool ends() const { return s + n == t.steps; }
  __device__ __forceinline__ int number() const { return CHOSEN ? t.number : t.row0 / ROWS; }
  __device__ __forceinline__ int pair(int tiles) const { return t.b * tiles + number(); }
  // Rows of the last V tile from `keep` on lie past the last key.
  __device__ __forceinline__ int keep() const { return t.kr.hi_max - t.kr.template key0<STEP>(s + n - 1); }
};

// Finds the block's share, with all threads; scratch: 16 64-bit words of shared memory.
template <int ROWS, int STEP, int COST, int THREADS, bool CHOSEN = false>
__device__ Share find_share(const AttendArgs& a, int tiles, int64_t* scratch) {
  const int pairs = a.p.n_seqs * tiles, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  constexpr int kWarps = THREADS / 32;
  if (CHOSEN && a.unit == kInTurn) {
    Share w = {};
    w.left = 1;  // to be walked; there may be nothing
    return w;
  }
  auto weight = [&](int p) {
    const int steps = p < pairs ? tile_of<ROWS, STEP, CHOSEN>(a, tiles, p).steps : 0;
    return steps > 0 ? static_cast<int64_t>(steps + COST) * a.p.heads : int64_t{0};
  };
  if (a.unit == 0) {
    const int item = static_cast<int>(blockIdx.x) / a.cluster, rank = static_cast<int>(blockIdx.x) - item * a.cluster;
    Share w;
    w.p = item / a.p.heads;
    w.head = item - w.p * a.p.heads;
    const int steps = tile_of<ROWS, STEP, CHOSEN>(a, tiles, w.p).steps;
    const int64_t from = static_cast<int64_t>(steps) * rank / a.cluster, to = static_cast<int64_t>(steps) * (rank + 1) / a.cluster;
    w.at = from > 0 ? from + COST : 0;
    w.left = to > from ? to + COST - w.at : 0;
    return w;
  }
  if (pairs <= 32) {  // every warp finds it by itself
    const int64_t mine = weight(lane);
    int64_t upto = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int64_t y = __shfl_up_sync(0xffffffffu, upto, d);
      if (lane >= d) upto += y;
    }
    const int64_t total = __shfl_sync(0xffffffffu, upto, 31);
    const int64_t per = max(divide(total + gridDim.x - 1, gridDim.x), static_cast<int64_t>(a.unit)), from = per * blockIdx.x;
    Share w;
    w.left = min(per, total - from);
    w.p = w.head = 0;
    w.at = 0;
    if (w.left > 0) {
      w.p = __ffs(__ballot_sync(0xffffffffu, from < upto)) - 1;
      const int64_t one = divide(__shfl_sync(0xffffffffu, mine, w.p), a.p.heads);
      const int64_t off = from - __shfl_sync(0xffffffffu, upto - mine, w.p);
      w.head = static_cast<int>(divide(off, one));
      w.at = off - w.head * one;
    }
    return w;
  }
  const int64_t first = weight(threadIdx.x);
  int64_t sum = first;
  for (int p = threadIdx.x + THREADS; p < pairs; p += THREADS) sum += weight(p);
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  if (lane == 0) scratch[warp] = sum;
  __syncthreads();
  int64_t total = 0;
#pragma unroll
  for (int i = 0; i < kWarps; ++i) total += scratch[i];
  int64_t per = divide(total + gridDim.x - 1, gridDim.x);
  if (per < a.unit) per = a.unit;
  const int64_t from = per * blockIdx.x;
  Share w;
  w.left = min(per, total - from);
  w.p = w.head = 0;
  w.at = 0;
  __syncthreads();
  if (w.left <= 0) return w;
  int64_t before = 0;
  for (int p0 = 0; p0 < pairs; p0 += THREADS) {
    const int64_t mine = p0 == 0 ? first : weight(p0 + threadIdx.x);
    int64_t upto = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int64_t y = __shfl_up_sync(0xffffffffu, upto, d);
      if (lane >= d) upto += y;
    }
    if (lane == 31) scratch[warp] = upto;
    __syncthreads();
    int64_t start = before, all = before;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) {
      if (i < warp) start += scratch[i];
      all += scratch[i];
    }
    start += upto - mine;
    if (from >= start && from < start + mine) {
      const int64_t one = divide(mine, a.p.heads), head = divide(from - start, one);
      scratch[kWarps] = p0 + threadIdx.x;
      scratch[kWarps + 1] = head;
      scratch[kWarps + 2] = from - start - head * one;
    }
    __syncthreads();
    if (from < all) break;
    before = all;
  }
  w.p = static_cast<int>(scratch[kWarps]);
  w.head = static_cast<int>(scratch[kWarps + 1]);
  w.at = scratch[kWarps + 2];
  return w;
}

// A record of a part: (0, pair of sequence and tile, KV head, these bits); all 0: no part.
enum : int { kPart = 4, kStarts = 1, kEnds = 2 };
__device__ __forceinline__ int4 part_record(int pair, int head, bool starts, bool ends) {
  return make_int4(0, pair, head, kPart | (starts ? kStarts : 0) | (ends ? kEnds : 0));
}

// The parts of the tile that block c starts and does not end, as whole warps:
// their number, 0 if there is none or if one is missing because its block gave up.
// Part 0 is slot `slot` (its record: rec), part i the first slot of block c + i.
__device__ __forceinline__ int parts_from(const AttendArgs& a, int c, int blocks, int& slot, int4& rec) {
  const int lane = threadIdx.x & 31;
  const int4 one = a.part_rec[2 * c], two = a.part_rec[2 * c + 1];
  int next = c + 1 + lane >= blocks ? 0 : a.part_rec[2 * (c + 1 + lane)].w;  // the first 32 with the records
  slot = two.w == (kPart | kStarts) ? 2 * c + 1 : one.w == (kPart | kStarts) ? 2 * c : -1;
  if (slot < 0) return 0;
  rec = slot & 1 ? two : one;
  for (int i0 = 1;; i0 += 32) {
    const uint32_t last = __ballot_sync(0xffffffffu, next != kPart);  // does not go on
    if (last) {
      const int at = __ffs(last) - 1;
      return __shfl_sync(0xffffffffu, next, at) == (kPart | kEnds) ? i0 + at + 1 : 0;
    }
    const int block = c + i0 + 32 + lane;
    next = block >= blocks ? 0 : a.part_rec[2 * block].w;
  }
}

}  // namespace ipv
