// sdv_tree_rows_d128.cu - the tree attention's kernels of many rows for heads of 128 elements.
#include "sdv_tree_rows.cuh"

namespace sdv {
cudaError_t launch_tree_rows_128(const AttendArgs& A, int rows, cudaStream_t s) { return launch_tree_rows<128>(TreeRowsArgs{A, rows, sm_count() / A.RT}, s); }
}  // namespace sdv
