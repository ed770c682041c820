// sdv_attend_d128.cu - the attention's kernels for heads of 128 elements.
#include "sdv_attend.cuh"

namespace sdv {
cudaError_t launch_attend_128(const AttendArgs& A, int nt, cudaStream_t s) { return launch_attend_d<128>(A, nt, s); }
}  // namespace sdv
