// kern_int8.cu -- product of 8-bit integers, S = a w^T, exact in int32, with scales
// per row and channel or as packed signs against thresholds.
//
// k_int8_plain: 64 rows x 64 channels per CTA, both operands' bytes of 64 k at a
// time in shared memory as words of four, dp4a.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "bmlp_internal.cuh"

namespace bk {
namespace {

// One scaled output (fp32 steps rounded one by one) or the sum itself.
__device__ __forceinline__ void store_out(const Int8Args& A, int64_t i, int j, int s) {
  const int64_t at = i * A.ldo + j;
  if (A.type == BMLP_I32) {
    static_cast<int32_t*>(A.out)[at] = s;
    return;
  }
  float y = (float)s;
  if (A.a_scale) y = __fmul_rn(y, A.a_scale[i]);
  if (A.w_scale) y = __fmul_rn(y, A.w_scale[j]);
  if (A.bias) y = __fadd_rn(y, A.bias[j]);
  if (A.type == BMLP_F32) static_cast<float*>(A.out)[at] = y;
  else if (A.type == BMLP_F16) static_cast<__half*>(A.out)[at] = __float2half_rn(y);
  else static_cast<__nv_bfloat16*>(A.out)[at] = __float2bfloat16_rn(y);
}

constexpr int PT = 64;       // tile
constexpr int kPThreads = 256;

__global__ void __launch_bounds__(kPThreads) k_int8_plain(const Int8Args A) {
  __shared__ int sa[16][PT + 1], sw[16][PT + 1];   // [word of four k][row]
  __shared__ uint32_t bits[PT][2];
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int j0 = (int)blockIdx.x * PT;
  const int64_t tiles = (A.n + PT - 1) / PT;
  for (int64_t t = blockIdx.y; t < tiles; t += gridDim.y) {
    const int64_t i0 = t * PT;
    int acc[4][4] = {};
    for (int k0 = 0; k0 < A.K; k0 += 64) {
      for (int e = threadIdx.x; e < PT * 16; e += kPThreads) {
        const int r = e >> 4, c = e & 15;
        uint32_t va = 0u, vw = 0u;
        for (int b = 0; b < 4; ++b) {
          const int k = k0 + 4 * c + b;
          if (k < A.K && i0 + r < A.n) va |= (uint32_t)(uint8_t)A.a[(i0 + r) * A.lda + k] << (8 * b);
          if (k < A.K && j0 + r < A.N) vw |= (uint32_t)(uint8_t)A.w[(j0 + r) * A.ldw + k] << (8 * b);
        }
        sa[c][r] = (int)va;
        sw[c][r] = (int)vw;
      }
      __syncthreads();
      for (int c = 0; c < 16; ++c)
        for (int u = 0; u < 4; ++u)
          for (int v = 0; v < 4; ++v) acc[u][v] = __dp4a(sa[c][ty + 16 * u], sw[c][tx + 16 * v], acc[u][v]);
      __syncthreads();
    }
    if (A.words) {
      if (threadIdx.x < 2 * PT) bits[threadIdx.x >> 1][threadIdx.x & 1] = 0u;
      __syncthreads();
      for (int u = 0; u < 4; ++u)
        for (int v = 0; v < 4; ++v) {
          const int j = j0 + tx + 16 * v;
          if (j < A.N && acc[u][v] >= (A.thr ? A.thr[j] : 0))
            atomicOr(&bits[ty + 16 * u][(tx + 16 * v) >> 5], 1u << ((tx + 16 * v) & 31));
        }
      __syncthreads();
      if (threadIdx.x < PT && i0 + threadIdx.x < A.n)
        A.words[(i0 + threadIdx.x) * ((A.N + 63) / 64) + blockIdx.x] =
            bits[threadIdx.x][0] | ((uint64_t)bits[threadIdx.x][1] << 32);
      __syncthreads();
    } else {
      for (int u = 0; u < 4; ++u)
        for (int v = 0; v < 4; ++v) {
          const int64_t i = i0 + ty + 16 * u;
          const int j = j0 + tx + 16 * v;
          if (i < A.n && j < A.N) store_out(A, i, j, acc[u][v]);
        }
    }
  }
}

}  // namespace

cudaError_t launch_int8(const Int8Args& A, cudaStream_t st) {
  const int64_t tiles = (A.n + PT - 1) / PT;
  const dim3 grid((unsigned)((A.N + PT - 1) / PT), (unsigned)(tiles < 65535 ? tiles : 65535));
  k_int8_plain<<<grid, kPThreads, 0, st>>>(A);
  return cudaGetLastError();
}

}  // namespace bk
