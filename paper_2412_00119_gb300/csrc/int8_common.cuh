// int8_common.cuh -- what the kernels of the 8-bit product share: reading a row's
// codes at any alignment, codes to fp16, and the scaled output.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "bmlp_internal.cuh"

namespace bk {
namespace i8 {

// One scaled output before its bias, fp32 steps rounded one by one; sa, sw: 1 where
// there is none.
__device__ __forceinline__ float scaled(int s, float sa, float sw) {
  return __fmul_rn(__fmul_rn((float)s, sa), sw);
}

template <typename T> __device__ __forceinline__ T out_cast(float y);
template <> __device__ __forceinline__ float out_cast(float y) { return y; }
template <> __device__ __forceinline__ __half out_cast(float y) { return __float2half_rn(y); }
template <> __device__ __forceinline__ __nv_bfloat16 out_cast(float y) { return __float2bfloat16_rn(y); }

__device__ __forceinline__ uint32_t skew_of(const int8_t* row) {
  return (uint32_t)(reinterpret_cast<uintptr_t>(row) & 3);
}

// Asynchronous copy of bytes [k, k + 16) of the K codes at row to shared memory, zeros
// from K on (k a multiple of 16; any: an address to name where nothing is read).  Rows
// that allow no 16-byte copies: the five aligned words around them.  Nothing past the
// row's K codes is read, and before them at most the rest of the first one's aligned
// word, which lies in the same allocation.
template <int kAlign>
__device__ __forceinline__ void copy16(uint32_t to, const int8_t* row, int k, int K, const int8_t* any) {
  if constexpr (kAlign == 16) {
    const int size = min(16, max(0, K - k));
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;"
                 ::"r"(to), "l"(size > 0 ? row + k : any), "r"(size) : "memory");
  } else {
    const int skew = (int)skew_of(row);
    const int8_t* p = row + (k - skew);
#pragma unroll
    for (int i = 0; i < 5; ++i) {
      const int size = K > 0 ? min(4, max(0, K - k + skew - 4 * i)) : 0;
      asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;"
                   ::"r"(to + 4u * i), "l"(size > 0 ? p + 4 * i : any - skew_of(any)), "r"(size) : "memory");
    }
  }
}

// Those sixteen codes back from shared memory, in the row's byte order.
template <int kAlign>
__device__ __forceinline__ void piece16(uint32_t (&v)[4], uint32_t from, const int8_t* row) {
  if constexpr (kAlign == 16) {
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(from) : "memory");
  } else {
    uint32_t w[5];
#pragma unroll
    for (int i = 0; i < 5; ++i) asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w[i]) : "r"(from + 4u * i) : "memory");
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __funnelshift_r(w[i], w[i + 1], 8u * skew_of(row));
  }
}

// Four codes as fp16: a code's byte with its sign bit flipped is code + 128, under the
// exponent of 1024 in a half's low byte it is 1152 + code, exactly.
__device__ __forceinline__ void codes_f16(uint32_t x, uint32_t& lo, uint32_t& hi) {
  const uint32_t u = x ^ 0x80808080u;
  const __half2 off = __halves2half2(__ushort_as_half(0x6480), __ushort_as_half(0x6480));   // 1152
  const uint32_t a = __byte_perm(u, 0x64646464u, 0x4140), b = __byte_perm(u, 0x64646464u, 0x4342);
  const __half2 ha = __hsub2(*reinterpret_cast<const __half2*>(&a), off);
  const __half2 hb = __hsub2(*reinterpret_cast<const __half2*>(&b), off);
  lo = *reinterpret_cast<const uint32_t*>(&ha);
  hi = *reinterpret_cast<const uint32_t*>(&hb);
}

// The call's rows from `rows` on.
inline Int8Args rest_of(Int8Args A, int64_t rows) {
  const int size = A.type == BMLP_F32 || A.type == BMLP_I32 ? 4 : 2;
  A.n -= rows;
  A.a += rows * A.lda;
  if (A.a_scale) A.a_scale += rows;
  if (A.out) A.out = static_cast<uint8_t*>(A.out) + rows * A.ldo * size;
  if (A.words) A.words += rows * ((A.N + 63) / 64);
  return A;
}

// 16: every row of both operands allows 16-byte loads; else 1.
inline int operand_align(const Int8Args& A) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(A.a) | (A.n > 1 ? (uintptr_t)A.lda : 0) |
                      reinterpret_cast<uintptr_t>(A.w) | (A.N > 1 ? (uintptr_t)A.ldw : 0);
  return (a & 15) == 0 ? 16 : 1;
}

}  // namespace i8
}  // namespace bk
