// sdv_attend_d64.cu - the attention's kernels for heads of 64 elements.
#include "sdv_attend.cuh"

namespace sdv {
cudaError_t launch_attend_64(const AttendArgs& A, int nt, cudaStream_t s) { return launch_attend_d<64>(A, nt, s); }
}  // namespace sdv
