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
__device__ __forceinline__ float scaled(float s, float sa, float sw) { return __fmul_rn(__fmul_rn(s, sa), sw); }

template <typename T> __device__ __forceinline__ T out_cast(float y);
template <> __device__ __forceinline__ float out_cast(float y) { return y; }
template <> __device__ __forceinline__ __half out_cast(float y) { return __float2half_rn(y); }
template <> __device__ __forceinline__ __nv_bfloat16 out_cast(float y) { return __float2bfloat16_rn(y); }

// Rows that allow no 16-byte copies (kAlign 1) are copied as the aligned 16-byte chunks
// around them: chunk i holds codes 16 i - s .. + 15, s the bytes between the row's start and
// the aligned address before it, and the codes [16 i, 16 i + 16) are merged from chunks i and i + 1.
template <int kAlign>
__device__ __forceinline__ int row_shift(const int8_t* row) {
  return kAlign == 16 ? 0 : (int)(reinterpret_cast<uintptr_t>(row) & 15);
}

// Asynchronous copy of the chunk that starts at code k (a multiple of 16) of the row's
// aligned chunks to shared memory, zeros from code K on; dead: K = -16.  Nothing past the
// row's K codes is read, and before them at most the rest of the first one's aligned 16
// bytes, which lie in the same allocation.  any: an address to name where nothing is read.
__device__ __forceinline__ void copy_chunk(uint32_t to, const int8_t* row, int shift, int k, int K, const int8_t* any) {
  const int size = min(16, max(0, K - k + shift));
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;"
               ::"r"(to), "l"(size > 0 ? row + (k - shift) : any), "r"(size) : "memory");
}
__device__ __forceinline__ const int8_t* aligned16(const int8_t* p) {
  return reinterpret_cast<const int8_t*>(reinterpret_cast<uintptr_t>(p) & ~(uintptr_t)15);
}

__device__ __forceinline__ void lds_chunk(uint32_t (&v)[4], uint32_t from) {
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(from) : "memory");
}

// Sixteen codes from two neighbouring chunks of a row with that shift.
__device__ __forceinline__ void merge16(uint32_t (&v)[4], const uint32_t (&lo)[4], const uint32_t (&hi)[4], int shift) {
  const bool two = shift & 8, one = shift & 4;
  uint32_t t[6], u[5];
#pragma unroll
  for (int i = 0; i < 6; ++i) {
    const uint32_t a = i < 4 ? lo[i < 4 ? i : 0] : hi[i < 4 ? 0 : i - 4];
    const uint32_t b = i + 2 < 4 ? lo[i + 2 < 4 ? i + 2 : 0] : hi[i + 2 < 4 ? 0 : i - 2];
    t[i] = two ? b : a;
  }
#pragma unroll
  for (int i = 0; i < 5; ++i) u[i] = one ? t[i + 1] : t[i];
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = __funnelshift_r(u[i], u[i + 1], 8u * (uint32_t)(shift & 3));
}

// Codes [k, k + 16) of a row straight to registers, zeros from K on (k a multiple of 16); what is
// read around them: as by the copies above.
__device__ __forceinline__ uint4 load_chunk(const int8_t* row, int shift, int k, int K) {
  const int8_t* p = row + (k - shift);
  const int size = K - k + shift;
  if (size >= 16) return __ldg(reinterpret_cast<const uint4*>(p));
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    w[i] = 0u;
    if (size >= 4 * i + 4) {
      w[i] = __ldg(reinterpret_cast<const uint32_t*>(p) + i);
    } else {
#pragma unroll
      for (int b = 0; b < 3; ++b)
        if (size > 4 * i + b) w[i] |= (uint32_t)(uint8_t)__ldg(p + 4 * i + b) << (8 * b);
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// shift: row_shift<kAlign>(row).
template <int kAlign>
__device__ __forceinline__ void load16(uint32_t (&v)[4], const int8_t* row, int shift, int k, int K) {
  const uint4 a = load_chunk(row, shift, k, K);
  const uint32_t lo[4] = {a.x, a.y, a.z, a.w};
  if constexpr (kAlign == 16) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = lo[i];
  } else {
    const uint4 b = load_chunk(row, shift, k + 16, K);
    const uint32_t hi[4] = {b.x, b.y, b.z, b.w};
    merge16(v, lo, hi, shift);
  }
}
// The same where every chunk read lies inside the row.
template <int kAlign>
__device__ __forceinline__ void load16_inside(uint32_t (&v)[4], const int8_t* row, int shift, int k) {
  const uint4* p = reinterpret_cast<const uint4*>(row + (k - shift));
  const uint4 a = __ldg(p);
  const uint32_t lo[4] = {a.x, a.y, a.z, a.w};
  if constexpr (kAlign == 16) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = lo[i];
  } else {
    const uint4 b = __ldg(p + 1);
    const uint32_t hi[4] = {b.x, b.y, b.z, b.w};
    merge16(v, lo, hi, shift);
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

// One output: the sum itself, or scaled.
__device__ __forceinline__ void put_out(const Int8Args& A, int64_t i, int j, int s) {
  const int64_t at = i * A.ldo + j;
  if (A.type == BMLP_I32) {
    static_cast<int32_t*>(A.out)[at] = s;
    return;
  }
  float y = scaled((float)s, A.a_scale ? A.a_scale[i] : 1.0f, A.w_scale ? A.w_scale[j] : 1.0f);
  if (A.bias) y = __fadd_rn(y, A.bias[j]);
  if (A.type == BMLP_F32) static_cast<float*>(A.out)[at] = y;
  else if (A.type == BMLP_F16) static_cast<__half*>(A.out)[at] = out_cast<__half>(y);
  else static_cast<__nv_bfloat16*>(A.out)[at] = out_cast<__nv_bfloat16>(y);
}

// Sum of products of the codes [k0, k1) of two rows.
static __device__ __noinline__ int plain_sum(const int8_t* ar, const int8_t* wr, int k0, int k1) {
  int sum = 0;
  for (int k = k0; k < k1; ++k) sum += (int)ar[k] * (int)wr[k];
  return sum;
}

// Outputs of `rows` rows from i0 and `channels` (a multiple of 32, as j0) channels from
// j0 by the whole CTA on CUDA cores: only after a wait has expired.
static __device__ __noinline__ void plain_tile(const Int8Args& A, int64_t i0, int rows, int j0, int channels) {
  const int warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31, warps = (int)blockDim.x >> 5;
  const int words = channels / 32, nw32 = 2 * ((A.N + 63) / 64);
  for (int e = warp; e < rows * words; e += warps) {
    const int64_t i = i0 + e / words;
    const int j = j0 + 32 * (e % words) + lane;
    if (i >= A.n) return;
    const int s = j < A.N ? plain_sum(A.a + i * A.lda, A.w + (int64_t)j * A.ldw, 0, A.K) : 0;
    if (A.words) {
      const uint32_t w = __ballot_sync(0xffffffffu, j < A.N && s >= (A.thr ? A.thr[j] : 0));
      if (lane == 0 && (j >> 5) < nw32) reinterpret_cast<uint32_t*>(A.words)[i * nw32 + (j >> 5)] = w;
    } else if (j < A.N) {
      put_out(A, i, j, s);
    }
  }
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

// 16: every row of the weights (of both operands) allows 16-byte loads; else 1.
inline int operand_align_w(const Int8Args& A) {
  return ((reinterpret_cast<uintptr_t>(A.w) | (A.N > 1 ? (uintptr_t)A.ldw : 0)) & 15) == 0 ? 16 : 1;
}
inline int operand_align(const Int8Args& A) {
  const bool a = ((reinterpret_cast<uintptr_t>(A.a) | (A.n > 1 ? (uintptr_t)A.lda : 0)) & 15) == 0;
  return a ? operand_align_w(A) : 1;
}

}  // namespace i8
}  // namespace bk
