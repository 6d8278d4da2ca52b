// kern_quantize.cu -- rows of real values to 8-bit codes and a scale per row, with
// or without the root-mean-square norm and the residual's addition before them.
//
//   h = x + res,  u = h gain,  A = max |u|,  rstd = 1 / sqrt(mean h^2 + eps)
//   q = rint(u (127 / A)),  scale = (A / 127) rstd
//
// rstd is common to a row, so the codes need A alone: the two reductions of a row,
// its sum of squares and its maximum, are made together, and every code is three
// rounded fp32 operations on its inputs (no contraction), the same in any layout.
// The maximum is taken on the bits of |u| as unsigned integers, whose order is the
// values' order with infinities and NaNs on top: one comparison finds those too.
//
// A CTA per row: the values are read twice (the second time from L1 or L2).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "bmlp_internal.cuh"

namespace bk {
namespace {

constexpr unsigned kFullMask = 0xffffffffu;
constexpr uint32_t kInfBits = 0x7F800000u;
constexpr float kLeast = 127.0f * 1.17549435e-38f;   // below it 127 / A leaves fp32's range

template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32(float v) { return v; }
template <> __device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
template <> __device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32(float v) { return v; }
template <> __device__ __forceinline__ __half from_f32(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32(float v) { return __float2bfloat16_rn(v); }

// The row's code factor and scale from the bits of A and (norm) its sum of squares.
struct RowScale {
  float inv, scale;
};
__device__ __forceinline__ RowScale row_scale(uint32_t abits, float sumsq, int K, float eps, bool norm) {
  RowScale r = {0.0f, __uint_as_float(0x7FFFFFFFu)};
  if (abits >= kInfBits || (norm && !(sumsq < __uint_as_float(kInfBits)))) return r;
  const float A = __uint_as_float(abits);
  r.scale = 0.0f;
  if (A < kLeast) return r;
  r.inv = 127.0f / A;
  r.scale = A / 127.0f;
  if (norm) r.scale = __fmul_rn(r.scale, 1.0f / sqrtf(__fadd_rn(sumsq / (float)K, eps)));
  return r;
}

// A value's code; inv == 0 (nothing to code, or a row that is not finite): 0.
__device__ __forceinline__ int code(float u, float inv) {
  const float c = inv == 0.0f ? 0.0f : __fmul_rn(u, inv);
  return min(127, max(-127, __float2int_rn(c)));
}

constexpr int kThreads = 256;

template <typename T, bool kNorm>
__global__ void __launch_bounds__(kThreads) k_quantize(const QuantArgs A) {
  __shared__ float ssum[kThreads / 32];
  __shared__ uint32_t smax[kThreads / 32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const T* gain = static_cast<const T*>(A.gain);
  for (int64_t row = blockIdx.x; row < A.n; row += gridDim.x) {
    const T* x = static_cast<const T*>(A.x) + row * A.ldx;
    const T* res = kNorm && A.res ? static_cast<const T*>(A.res) + row * A.ldr : nullptr;
    T* sum = kNorm && A.sum ? static_cast<T*>(A.sum) + row * A.lds : nullptr;
    auto h_of = [&](int i) { return res ? __fadd_rn(to_f32(x[i]), to_f32(res[i])) : to_f32(x[i]); };
    auto u_of = [&](float h, int i) { return kNorm && gain ? __fmul_rn(h, to_f32(gain[i])) : h; };
    float sq = 0.0f;
    uint32_t most = 0u;
    for (int i = threadIdx.x; i < A.K; i += kThreads) {
      const float h = h_of(i);
      sq += h * h;
      most = max(most, __float_as_uint(u_of(h, i)) & 0x7FFFFFFFu);
    }
    for (int o = 16; o > 0; o >>= 1) sq += __shfl_xor_sync(kFullMask, sq, o);
    most = __reduce_max_sync(kFullMask, most);
    if (lane == 0) {
      ssum[warp] = sq;
      smax[warp] = most;
    }
    __syncthreads();
    sq = 0.0f;
    most = 0u;
    for (int w = 0; w < kThreads / 32; ++w) {
      sq += ssum[w];
      most = max(most, smax[w]);
    }
    const RowScale r = row_scale(most, sq, A.K, A.eps, kNorm);
    // the row's values again: a thread writes its own elements of sum_out only after
    // it has read them (sum_out may be x or res)
    for (int i = threadIdx.x; i < A.K; i += kThreads) {
      const float h = h_of(i);
      if (sum) sum[i] = from_f32<T>(h);
      A.q[row * A.ldq + i] = (int8_t)code(u_of(h, i), r.inv);
    }
    if (threadIdx.x == 0) A.scale[row] = r.scale;
    __syncthreads();
  }
}

template <typename T>
cudaError_t launch_type(const QuantArgs& A, bool norm, cudaStream_t st) {
  const unsigned grid = (unsigned)(A.n < 65536 ? A.n : 65536);
  if (norm) k_quantize<T, true><<<grid, kThreads, 0, st>>>(A);
  else k_quantize<T, false><<<grid, kThreads, 0, st>>>(A);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_quantize(const QuantArgs& A, bool norm, cudaStream_t st) {
  switch (A.type) {
    case BMLP_F32: return launch_type<float>(A, norm, st);
    case BMLP_F16: return launch_type<__half>(A, norm, st);
    default: return launch_type<__nv_bfloat16>(A, norm, st);
  }
}

}  // namespace bk
