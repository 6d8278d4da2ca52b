// kern_mx4_product.cu -- product of microscaled 4-bit rows,
//   y_ij = row_scale_i sum_b 2^(sa_ib + sw_jb - 254) sum_{k in block b} a_ik w_jk + bias_j,
// with one matrix of weights or that of each row's group.
//
// k_mx4_plain: a thread per output (1 x 8192 -> 8192 576 us, 100 x 4096 -> 8192 6.3 ms).
#include <algorithm>

#include "mx4_common.cuh"

namespace bk {
namespace {

using namespace mx4;

constexpr int kThreads = 256;

__global__ void __launch_bounds__(kThreads) k_mx4_plain(const Mx4Args A) {
  pdl_wait();
  pdl_trigger();
  const int64_t total = A.n * A.N;
  for (int64_t t = (int64_t)blockIdx.x * kThreads + threadIdx.x; t < total; t += (int64_t)gridDim.x * kThreads) {
    const int64_t i = t / A.N;
    const int j = (int)(t % A.N);
    int e = 0;
    if (A.offsets) {
      // the last group that starts at or before the row
      int at = clamp_offset(A.offsets[0], 0, A.n);
      e = -1;
      for (int g = 0; g < A.E && e < 0; ++g) {
        const int end = clamp_offset(A.offsets[g + 1], at, A.n);
        if (i >= at && i < end) e = g;
        at = end;
      }
      if (e < 0) continue;
    }
    put_out(A, i, j, e, plain_sum(A, i, j, e));
  }
}

}  // namespace

cudaError_t launch_mx4(const Mx4Args& A, cudaStream_t st, int) {
  const int64_t ctas = (A.n * A.N + kThreads - 1) / kThreads;
  return launch_kernel(k_mx4_plain, dim3((unsigned)std::min<int64_t>(ctas, 64ll * sm_count())), dim3(kThreads), 0, st, true, A);
}

}  // namespace bk
