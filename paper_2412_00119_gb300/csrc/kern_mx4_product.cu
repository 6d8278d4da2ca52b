// kern_mx4_product.cu -- product of microscaled 4-bit rows,
//   y_ij = row_scale_i sum_b 2^(sa_ib + sw_jb - 254) sum_{k in block b} a_ik w_jk + bias_j,
// with one matrix of weights or that of each row's group: the choice of kernel.
#include "bmlp_internal.cuh"

namespace bk {

cudaError_t launch_mx4(const Mx4Args& A, cudaStream_t st, int expire) { return launch_mx4_tile(A, st, expire); }

}  // namespace bk
