// mx4_common.cuh -- what the kernels of the microscaled 4-bit product share: the groups'
// rows, one output after its sum, and sums on CUDA cores.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "bmlp_internal.cuh"

namespace bk {
namespace mx4 {

// Map of rows of codes, box_rows of 128 bytes (256 codes) at a time in the 128B-swizzled order that
// the MMAs read; groups > 0: of groups of rows.  False where tensor copies cannot take them:
// rows or groups that do not start at multiples of 16 bytes.
inline bool code_map(CUtensorMap* map, const uint8_t* codes, int64_t bytes, int64_t rows, int64_t ld, int64_t groups,
                     int64_t group_ld, int box_rows) {
  typedef CUresult (*Encode)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                             const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                             CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  static const Encode encode = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess)
      f = nullptr;
    return reinterpret_cast<Encode>(f);
  }();
  const int64_t least = (bytes + 15) / 16 * 16;
  if (rows == 1) ld = least;                  // (a stride that nothing uses)
  if (groups <= 1) group_ld = least;
  if (!encode || ((reinterpret_cast<uintptr_t>(codes) | (uintptr_t)ld | (uintptr_t)group_ld) & 15) != 0 || group_ld == 0 ||
      ld >= (1ll << 40) || group_ld >= (1ll << 40))
    return false;
  const cuuint64_t dims[3] = {(cuuint64_t)bytes, (cuuint64_t)rows, (cuuint64_t)groups};
  const cuuint64_t strides[2] = {(cuuint64_t)ld, (cuuint64_t)group_ld};
  const cuuint32_t box[3] = {128, (cuuint32_t)box_rows, 1}, steps[3] = {1, 1, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, groups > 0 ? 3 : 2, const_cast<uint8_t*>(codes), dims, strides, box, steps,
                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Rows [first, last) of a group.  Offsets that decrease or leave 0..n are taken as the
// nearest that do not: callers pass the largest offset before as `low`.
__device__ __forceinline__ int clamp_offset(int32_t offset, int low, int64_t n) {
  return max(low, min((int)n, (int)offset));
}

template <typename T> __device__ __forceinline__ T out_cast(float y);
template <> __device__ __forceinline__ float out_cast(float y) { return y; }
template <> __device__ __forceinline__ __half out_cast(float y) { return __float2half_rn(y); }
template <> __device__ __forceinline__ __nv_bfloat16 out_cast(float y) { return __float2bfloat16_rn(y); }

// Product of two bytes of codes: the sum of two exact products (multiples of 1/4).
__device__ __forceinline__ float pair_product(uint32_t a, uint32_t b) {
  uint32_t x, y;
  asm("{\n .reg .b8 p;\n cvt.u8.u32 p, %1;\n cvt.rn.f16x2.e2m1x2 %0, p;\n}" : "=r"(x) : "r"(a));
  asm("{\n .reg .b8 p;\n cvt.u8.u32 p, %1;\n cvt.rn.f16x2.e2m1x2 %0, p;\n}" : "=r"(y) : "r"(b));
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&x)), g = __half22float2(*reinterpret_cast<const __half2*>(&y));
  return fmaf(f.x, g.x, f.y * g.y);
}

// Sum over K of row i against channel j of group e, block by block (a block's sum is exact).
static __device__ __noinline__ float plain_sum(const Mx4Args& A, int64_t i, int j, int e) {
  const uint8_t *a = A.a + i * A.lda, *as = A.as + i * A.ldas;
  const uint8_t *w = A.w + e * A.gw + j * A.ldw, *ws = A.ws + e * A.gws + j * A.ldws;
  const int64_t bytes = ((int64_t)A.K + 1) / 2;
  float sum = 0.0f;
  for (int64_t b = 0; 16 * b < bytes; ++b) {
    float s = 0.0f;
    for (int64_t k = 16 * b; k < min(bytes, 16 * b + 16); ++k) s += pair_product(a[k], w[k]);
    const uint32_t p = as[b], q = ws[b];
    sum += p == 255u || q == 255u ? __uint_as_float(0x7FFFFFFFu) : scalbnf(s, (int)(p + q) - 254);
  }
  return sum;
}

__device__ __forceinline__ void put_out(const Mx4Args& A, int64_t i, int j, int e, float sum) {
  float y = A.row_scale ? __fmul_rn(sum, A.row_scale[i]) : sum;
  if (A.bias) y = __fadd_rn(y, A.bias[e * A.ldb + j]);
  const int64_t at = i * A.ldo + j;
  if (A.type == BMLP_F32) static_cast<float*>(A.out)[at] = y;
  else if (A.type == BMLP_F16) static_cast<__half*>(A.out)[at] = out_cast<__half>(y);
  else static_cast<__nv_bfloat16*>(A.out)[at] = out_cast<__nv_bfloat16>(y);
}

}  // namespace mx4
}  // namespace bk
