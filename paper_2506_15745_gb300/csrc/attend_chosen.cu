// Attention of each new row over the pages that it has chosen, a list for each KV
// head (attend_rows.cuh).
#include "attend_rows.cuh"

namespace ipv {

int attend_chosen_resident(int fmt, int dim, int tile) { return resident<true>(fmt, dim, tile); }
cudaError_t attend_chosen_prepare() { return prepare<true>(); }
cudaError_t launch_attend_chosen(const AttendArgs& a, int blocks, cudaStream_t st) { return launch<true>(a, blocks, st); }

}  // namespace ipv
