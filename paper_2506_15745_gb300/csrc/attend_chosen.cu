// Attention of each new row over the pages that it has chosen, a list for each KV
// head: the rows kernel (attend_rows.cuh) with tiles of one new row's query heads,
// keys that count through the row's list, and look-ups of 16 steps at once. What bounds it:
// HBM for tokens of many streams over bf16 pages (48 streams, 64 pages of 32 rows, 403 MB: 64 us, 6.3 TB/s); L2 and the
// chain of a step for questions, whose rows read the same pages (8 streams of up to 61 tokens: 67 us, 13 TB/s out
// of L2 for 137 MB of distinct pages); the instructions of a step over 4-bit pages (32 streams, 77 MB: 27 us); the chain
// of look-ups, one step and the join for one token (32 pages: 7.1 us).
#include "attend_rows.cuh"

namespace ipv {

int attend_chosen_resident(int fmt, int dim, int tile) { return resident<true>(fmt, dim, tile); }
cudaError_t attend_chosen_prepare() { return prepare<true>(); }
cudaError_t launch_attend_chosen(const AttendArgs& a, int blocks, cudaStream_t st) { return launch<true>(a, blocks, st); }

}  // namespace ipv
