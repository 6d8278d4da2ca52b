// kern_int8.cu -- product of 8-bit integers, S = a w^T, exact in int32, with scales
// per row and channel or as packed signs against thresholds: the choice of kernel.
#include "int8_common.cuh"

namespace bk {

cudaError_t launch_int8(const Int8Args& A, cudaStream_t st) { return launch_int8_tile(A, st, 0); }

}  // namespace bk
