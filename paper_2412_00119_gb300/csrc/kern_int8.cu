// kern_int8.cu -- product of 8-bit integers, S = a w^T, exact in int32, with scales
// per row and channel or as packed signs against thresholds: the choice of kernel.
#include "bmlp_internal.cuh"

namespace bk {

int64_t int8_workspace(int64_t n, int K, int N) {
  // (blocks are numbered in 31 bits)
  return n >= 256 && ((int64_t)N + 256) * (K / 64 + 1) < (1ll << 31) ? int8_pair_workspace(n, K, N) : 0;
}

cudaError_t launch_int8(const Int8Args& A, void* workspace, int64_t workspace_bytes, cudaStream_t st) {
  if (A.n <= kFewRows) return launch_int8_few(A, st);
  const int64_t want = int8_workspace(A.n, A.K, A.N);
  if (want > 0 && workspace && workspace_bytes >= want) return launch_int8_pair(A, workspace, st, 0);
  return launch_int8_tile(A, st, 0);
}

}  // namespace bk
