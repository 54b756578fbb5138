// Attention of each new row over the pages that it has chosen, a list for each KV
// head: the rows kernel (attend_rows.cuh) with tiles of one new row's query heads,
// keys that count through the row's list, and look-ups of 16 steps at once. What bounds it:
// HBM for tokens of many streams over bf16 pages (48 streams, 64 pages of 32 rows, 403 MB: 64 us, 6.3 TB/s); L2 and the
// chain of a step for questions, whose rows read the same pages (8 streams of up to 61 tokens: 66 us, 13 TB/s out
// of L2 for 137 MB of distinct pages). Over codes a page is unpacked again for each row that chose it, twice the
// instructions of bf16 (46 and 57 million against 28): the same questions 77 us over 4 bits, 96 over 8. Few tokens over 4-bit
// pages wait: 32 streams (77 MB, 27 us) leave 8 warps on two thirds of the SMs and 4 on the others, issue is active 41%.
// One token (32 pages: 7.1 us) is the chain of look-ups, one step and the join.
#include "attend_rows.cuh"

namespace ipv {

int attend_chosen_resident(int fmt, int dim, int tile) { return resident<true>(fmt, dim, tile); }
cudaError_t attend_chosen_prepare() { return prepare<true>(); }
cudaError_t launch_attend_chosen(const AttendArgs& a, int blocks, cudaStream_t st) { return launch<true>(a, blocks, st); }

}  // namespace ipv
