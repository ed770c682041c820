// sdv_tree_attend_d64.cu - the tree attention's kernels of few rows for heads of 64 elements.
#include "sdv_attend.cuh"

namespace sdv {
cudaError_t launch_tree_attend_64(const AttendArgs& A, int nt, cudaStream_t s) { return launch_attend_d<64, true>(A, nt, s); }
}  // namespace sdv
