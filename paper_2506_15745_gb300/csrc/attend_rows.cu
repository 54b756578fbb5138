// Attention of a few query rows over all the rows that they see (attend_rows.cuh).
#include "attend_rows.cuh"

namespace ipv {

int attend_rows_tile(int rows) { return rows <= 8 ? 8 : 16; }
int attend_rows_resident(int fmt, int dim, int tile) { return resident<false>(fmt, dim, tile); }
cudaError_t attend_rows_prepare() { return prepare<false>(); }
cudaError_t launch_attend_rows(const AttendArgs& a, int blocks, cudaStream_t st) { return launch<false>(a, blocks, st); }

}  // namespace ipv
