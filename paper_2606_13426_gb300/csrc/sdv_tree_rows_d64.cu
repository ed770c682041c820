// sdv_tree_rows_d64.cu - the tree attention's kernels of many rows for heads of 64 elements.
#include "sdv_tree_rows.cuh"

namespace sdv {
cudaError_t launch_tree_rows_64(const AttendArgs& A, int rows, cudaStream_t s) { return launch_tree_rows<64>(TreeRowsArgs{A, rows, sm_count() / A.RT}, s); }
}  // namespace sdv
