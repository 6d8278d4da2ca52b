// kern_mx4_quantize.cu -- rows of real values to microscaled 4-bit codes (e2m1, two to a
// byte, with a power-of-two scale per 32), with or without the root-mean-square norm
// and the residual's addition before them, and codes back to real values.
//
//   h = x + res,  u = h gain,  of each 32 u: m = max |u|,
//   s = max(0, floor(log2 m) - 2 + 127),  code = e2m1(u 2^(127-s)),  row_scale = 1 / sqrt(mean h^2 + eps)
//
// 2^(127-s) is a normal fp32 number for every finite m, and the product with it exact, so a
// code has one rounding (and u at most two).  The norm's factor stays outside of the
// codes: they need their own 32 values alone, and a row passes through once, whatever its
// length, with the sum of squares running beside.  The maximum is taken on the bits of |u| as
// unsigned integers, whose order is the values' order with infinities and NaNs on top.
// Bound: memory, and the instructions beside it.  8192 x 8192 bf16 34 us (5.0 TB/s), back to values 26 (6.5), the
// norm of 8191 x 4096 bf16 with residual 37 (6.0); 24,095 x 787 fp32, rows at odd places, 22, 23 and 51.
#include <algorithm>
#include <type_traits>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "bmlp_internal.cuh"

namespace bk {
namespace {

constexpr unsigned kFullMask = 0xffffffffu;
constexpr uint32_t kInfBits = 0x7F800000u;

// A value's bits in type T.  Rows are read and written as bits, with the same types for both: a sum may be
// stored where its row was read, and accesses of different types may change places in a compiler's hands.
template <typename T> struct Bits { typedef uint16_t Type; };
template <> struct Bits<float> { typedef uint32_t Type; };
template <typename T> __device__ __forceinline__ typename Bits<T>::Type bits_of(float v);
template <> __device__ __forceinline__ uint32_t bits_of<float>(float v) { return __float_as_uint(v); }
template <> __device__ __forceinline__ uint16_t bits_of<__half>(float v) { return __half_as_ushort(__float2half_rn(v)); }
template <> __device__ __forceinline__ uint16_t bits_of<__nv_bfloat16>(float v) { return __bfloat16_as_ushort(__float2bfloat16_rn(v)); }

// Below this eps (2^-80) a row's factor may hang on squares that are lost in fp32, those of
// |h| < 2^-63.  Such rows have a sum below kSmallSum (2^-90: what a greater one has lost is
// less than 2^-60 of it for each value), every |h| below 2^-45, and squares of h kUp (2^85)
// that are inside fp32's range down to its least subnormal.
constexpr float kSmallEps = 8.27180613e-25f, kSmallSum = 8.07793566e-28f;
constexpr float kUp = 3.86856262e25f;   // 2^85

__device__ __forceinline__ float row_factor(float sumsq, float sumsq_up, int K, float eps, bool small) {
  if (!(sumsq < __uint_as_float(kInfBits))) return __uint_as_float(0x7FFFFFFFu);
  const bool up = small && sumsq < kSmallSum;
  const float root = up ? sqrtf(sumsq_up / (float)K + eps * kUp * kUp) : sqrtf(sumsq / (float)K + eps);
  return root > 0.0f ? (up ? (1.0f / root) * kUp : 1.0f / root) : 0.0f;
}

// The 32 bits at word i of a vector of them.
template <typename T, int V>
__device__ __forceinline__ uint32_t word_of(const float (&f)[V], int i) {
  if constexpr (std::is_same<T, float>::value) {
    return __float_as_uint(f[i]);
  } else if constexpr (std::is_same<T, __half>::value) {
    const __half2 h = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
    return *reinterpret_cast<const uint32_t*>(&h);
  } else {
    const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
}

// V values, of 16 bytes or of 8, as they lie in memory (wide: 16, aligned).
template <typename T, int V, bool kWide = true> struct Values {
  static constexpr int kWords = V * (int)sizeof(T) / 4;
  static_assert(kWide ? kWords == 4 : kWords == 4 || kWords == 2, "whole words");
  uint32_t w[kWords];
  // the first `left` of those at p; zeros in the others' place
  __device__ __forceinline__ void load(const T* p, int64_t left) {
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = 0u;
    if constexpr (kWide) {
      if (left >= V) {
        const uint4 v = *reinterpret_cast<const uint4*>(p);
        w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
        return;
      }
    }
    // one by one: the lines stay in L1 meanwhile
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < left) {
        if constexpr (sizeof(T) == 4) w[i] = *reinterpret_cast<const uint32_t*>(p + i);
        else w[i / 2] |= (uint32_t)*reinterpret_cast<const uint16_t*>(p + i) << (16 * (i % 2));
      }
  }
  // The bits, as fp32, of the largest |value|.  (The order of |values| is that of their bits, in each type.)
  __device__ __forceinline__ uint32_t most() const {
    if constexpr (std::is_same<T, float>::value) {
      uint32_t m = 0u;
#pragma unroll
      for (int i = 0; i < kWords; ++i) m = max(m, w[i] & 0x7FFFFFFFu);
      return m;
    } else {
      uint32_t m = 0u;
#pragma unroll
      for (int i = 0; i < kWords; ++i) m = __vmaxu2(m, w[i] & 0x7FFF7FFFu);
      m = max(m & 0xFFFFu, m >> 16);
      if constexpr (std::is_same<T, __half>::value) return __float_as_uint(__half2float(__ushort_as_half((unsigned short)m)));
      else return m << 16;
    }
  }
  __device__ __forceinline__ float get(int i) const {
    if constexpr (std::is_same<T, float>::value) return __uint_as_float(w[i]);
    else if constexpr (std::is_same<T, __half>::value) return __half2float(__ushort_as_half((unsigned short)(w[i / 2] >> (16 * (i % 2)))));
    else return __uint_as_float(i % 2 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
  }
};

template <typename T, int V, bool kWide = true>
__device__ __forceinline__ void store_values(T* p, const float (&f)[V], int64_t left) {
  if constexpr (kWide) {
    if (left >= V) {
      constexpr int kWords = V * (int)sizeof(T) / 4;
      static_assert(kWords % 4 == 0, "whole vectors");
#pragma unroll
      for (int i = 0; i < kWords; i += 4)
        *reinterpret_cast<uint4*>(p + 4 * i / (int)sizeof(T)) =
            make_uint4(word_of<T>(f, i), word_of<T>(f, i + 1), word_of<T>(f, i + 2), word_of<T>(f, i + 3));
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < V; ++i)
    if (i < left) reinterpret_cast<typename Bits<T>::Type*>(p)[i] = bits_of<T>(f[i]);
}

// Two codes in a byte, ties to the even code.
__device__ __forceinline__ uint32_t code_pair(float lo, float hi) {
  uint32_t r;
  asm("{\n .reg .b8 b;\n cvt.rn.satfinite.e2m1x2.f32 b, %1, %2;\n cvt.u32.u8 %0, b;\n}" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// Bits of the largest |u|.
template <int V>
__device__ __forceinline__ uint32_t largest(const float (&u)[V]) {
  uint32_t m = 0u;
#pragma unroll
  for (int i = 0; i < V; ++i) m = max(m, __float_as_uint(u[i]) & 0x7FFFFFFFu);
  return m;
}
// Codes of a lane's V values u and their block's scale byte s; m: bits of the lane's largest |u|.  Blocks of 32 are
// 32 / V neighbouring lanes'; every lane of the warp calls.
template <int V>
__device__ __forceinline__ uint32_t make_codes(const float (&u)[V], uint32_t m, uint32_t& s) {
  static_assert(V == 4 || V == 8, "a lane's values");
#pragma unroll
  for (int o = 1; o < 32 / V; o *= 2) m = max(m, __shfl_xor_sync(kFullMask, m, o));
  const bool finite = m < kInfBits;
  const uint32_t e = m >> 23;
  s = finite ? (e > 2u ? e - 2u : 0u) : 255u;
  const float up = __uint_as_float(finite ? (254u - s) << 23 : 0u);
  uint32_t c = 0u;
#pragma unroll
  for (int i = 0; i < V; i += 2) c |= code_pair(u[i] * up, u[i + 1] * up) << (4 * i);
  return finite ? c : 0u;
}

// Codes and scale of a lane's V values from element e of a row on, `left` of which are the row's.
template <int V, bool kWide = true>
__device__ __forceinline__ void store_codes(uint8_t* q, uint8_t* scale, int64_t e, int64_t left, uint32_t c, uint32_t s) {
  const int lane = threadIdx.x & 31;
  if (kWide && left >= V) {
    if constexpr (V == 8) *reinterpret_cast<uint32_t*>(q + (e >> 1)) = c;
    else *reinterpret_cast<uint16_t*>(q + (e >> 1)) = (uint16_t)c;
  } else {
#pragma unroll
    for (int i = 0; i < V / 2; ++i)
      if (2 * i < left) q[(e >> 1) + i] = (uint8_t)(c >> (8 * i));
  }
  if (lane % (32 / V) == 0 && left > 0) scale[e >> 5] = (uint8_t)s;
}

// ---------------------------------------------------------------------------
// Without a norm: a warp takes kAhead times 32 V neighbouring values of a row at a time.
// ---------------------------------------------------------------------------
constexpr int kThreads = 256;

// Unit t of n rows of `parts` units.
__device__ __forceinline__ void unit_at(int64_t t, int64_t parts, bool narrow, int64_t& row, int64_t& part) {
  if (narrow) {   // (a 64-bit division takes as long as the rest of a unit)
    row = (uint32_t)t / (uint32_t)parts;
    part = (uint32_t)t - (uint32_t)row * (uint32_t)parts;
  } else {
    row = t / parts;
    part = t - row * parts;
  }
}

template <typename T, int V, bool kWideX, bool kWideQ, int kAhead>
__global__ void __launch_bounds__(kThreads, 5) k_mx4_quantize(const Mx4QuantArgs A) {
  pdl_wait();
  pdl_trigger();
  constexpr int kPart = 32 * V * kAhead;
  const int lane = threadIdx.x & 31;
  const int64_t parts = ((int64_t)A.K + kPart - 1) / kPart, total = A.n * parts;
  const bool narrow = total < (1ll << 31);
  for (int64_t t = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); t < total;
       t += (int64_t)gridDim.x * (kThreads / 32)) {
    int64_t row, part;
    unit_at(t, parts, narrow, row, part);
    const int64_t e0 = part * kPart + V * lane;
    const T* x = static_cast<const T*>(A.x) + row * A.ldx;
    Values<T, V, kWideX> v[kAhead];
#pragma unroll
    for (int a = 0; a < kAhead; ++a) v[a].load(x + e0 + 32 * V * a, A.K - (e0 + 32 * V * a));
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      const int64_t e = e0 + 32 * V * a;
      float u[V];
#pragma unroll
      for (int i = 0; i < V; ++i) u[i] = v[a].get(i);
      uint32_t s;
      const uint32_t c = make_codes<V>(u, v[a].most(), s);
      store_codes<V, kWideQ>(A.q + row * A.ldq, A.scale + row * A.ldc, e, A.K - e, c, s);
    }
  }
}

// ---------------------------------------------------------------------------
// With it: a row's threads are a warp (kWarpRow) or a CTA.
// ---------------------------------------------------------------------------
template <typename T, bool kRes, bool kSmall, int V, bool kWide, int kAhead, bool kWarpRow>
__global__ void __launch_bounds__(kWarpRow ? kThreads : 1024) k_mx4_norm(const Mx4QuantArgs A) {
  pdl_wait();
  pdl_trigger();
  const int threads = kWarpRow ? 32 : (int)blockDim.x, lane = threadIdx.x & 31;
  const int tid = kWarpRow ? lane : (int)threadIdx.x;
  const int64_t row = kWarpRow ? (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5) : (int64_t)blockIdx.x;
  if (kWarpRow && row >= A.n) return;
  const T* x = static_cast<const T*>(A.x) + row * A.ldx;
  const T* res = kRes ? static_cast<const T*>(A.res) + row * A.ldr : nullptr;
  T* sum = A.sum ? static_cast<T*>(A.sum) + row * A.lds : nullptr;
  const T* gain = static_cast<const T*>(A.gain);
  float sq = 0.0f, sq_up = 0.0f;
  const int64_t step = (int64_t)threads * V;
  // (whole warps: the lanes of one meet in make_codes)
  for (int64_t e0 = V * tid; e0 - V * lane < A.K; e0 += kAhead * step) {
    Values<T, V, kWide> v[kAhead], r[kRes ? kAhead : 1], g[kAhead];
#pragma unroll
    for (int a = 0; a < kAhead; ++a) v[a].load(x + e0 + a * step, A.K - (e0 + a * step));
    if constexpr (kRes) {
#pragma unroll
      for (int a = 0; a < kAhead; ++a) r[a].load(res + e0 + a * step, A.K - (e0 + a * step));
    }
    if (gain) {
#pragma unroll
      for (int a = 0; a < kAhead; ++a) g[a].load(gain + e0 + a * step, A.K - (e0 + a * step));
    }
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      const int64_t e = e0 + a * step, left = A.K - e;
      float u[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        u[i] = v[a].get(i);
        if constexpr (kRes) u[i] = __fadd_rn(u[i], r[a].get(i));
        sq += u[i] * u[i];
        if constexpr (kSmall) sq_up += (u[i] * kUp) * (u[i] * kUp);
      }
      // (these values of x and res are read: sum_out may be one of them)
      if (sum) store_values<T, V, kWide>(sum + e, u, left);
      if (gain) {
#pragma unroll
        for (int i = 0; i < V; ++i) u[i] = __fmul_rn(u[i], g[a].get(i));
      }
      uint32_t s;
      const uint32_t c = make_codes<V>(u, largest<V>(u), s);
      store_codes<V, kWide>(A.q + row * A.ldq, A.scale + row * A.ldc, e, left, c, s);
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    sq += __shfl_xor_sync(kFullMask, sq, o);
    if constexpr (kSmall) sq_up += __shfl_xor_sync(kFullMask, sq_up, o);
  }
  if constexpr (!kWarpRow) {
    __shared__ float part[2][32];
    const int warp = threadIdx.x >> 5, warps = (int)blockDim.x >> 5;
    if (lane == 0) {
      part[0][warp] = sq;
      part[1][warp] = sq_up;
    }
    __syncthreads();
    if (warp != 0) return;
    sq = lane < warps ? part[0][lane] : 0.0f;
    sq_up = lane < warps ? part[1][lane] : 0.0f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      sq += __shfl_xor_sync(kFullMask, sq, o);
      if constexpr (kSmall) sq_up += __shfl_xor_sync(kFullMask, sq_up, o);
    }
  }
  if (tid == 0) A.row_scale[row] = row_factor(sq, sq_up, A.K, A.eps, kSmall);
}

// ---------------------------------------------------------------------------
// Codes to values.
// ---------------------------------------------------------------------------
// The two values of a byte of codes.
__device__ __forceinline__ float2 pair_values(uint32_t byte) {
  uint32_t h;
  asm("{\n .reg .b8 b;\n cvt.u8.u32 b, %1;\n cvt.rn.f16x2.e2m1x2 %0, b;\n}" : "=r"(h) : "r"(byte));
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

// A warp takes kAhead times 32 V neighbouring codes of a row at a time: all its loads, then its stores.
template <typename T, int V, int kAhead>
__global__ void __launch_bounds__(kThreads) k_mx4_dequantize(const Mx4DequantArgs A) {
  pdl_wait();
  pdl_trigger();
  constexpr int kPart = 32 * V * kAhead;
  const int lane = threadIdx.x & 31;
  const int64_t parts = ((int64_t)A.K + kPart - 1) / kPart, total = A.n * parts;
  const bool narrow = total < (1ll << 31);
  for (int64_t t = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); t < total;
       t += (int64_t)gridDim.x * (kThreads / 32)) {
    int64_t row, part;
    unit_at(t, parts, narrow, row, part);
    const int64_t e0 = part * kPart + V * lane;
    const uint8_t *q = A.q + row * A.ldq, *scale = A.scale + row * A.ldc;
    uint32_t c[kAhead], s[kAhead];
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      const int64_t e = e0 + 32 * V * a, left = A.K - e;
      c[a] = 0u;
      s[a] = left > 0 ? scale[e >> 5] : 127u;
      if constexpr (V == 8) {
        if (left >= V - 1) {
          c[a] = *reinterpret_cast<const uint32_t*>(q + (e >> 1));
        } else {
#pragma unroll
          for (int i = 0; i < V / 2; ++i)
            if (2 * i < left) c[a] |= (uint32_t)q[(e >> 1) + i] << (8 * i);
        }
      } else {
        if (left > 0) c[a] = q[e >> 1];
      }
    }
    const float by = A.row_scale ? A.row_scale[row] : 1.0f;
    auto put = [&](int a, const float (&f)[V]) {
      const int64_t e = e0 + 32 * V * a;
      store_values<T, V, V == 8>(static_cast<T*>(A.out) + row * A.ldo + e, f, A.K - e);
    };
    // 2^(s-127) times the row's factor is exact where it is a normal number, and its product with a code the one
    // rounding.
    float unit[kAhead];
    bool plain = true;
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      unit[a] = __uint_as_float(s[a] << 23) * by;
      plain = plain && (__float_as_uint(unit[a]) & 0x7FFFFFFFu) - 0x00800000u < kInfBits - 0x00800000u;
    }
    if (__all_sync(kFullMask, plain)) {
#pragma unroll
      for (int a = 0; a < kAhead; ++a) {
        float f[V];
#pragma unroll
        for (int i = 0; i < V; i += 2) {
          const float2 two = pair_values((c[a] >> (4 * i)) & 255u);
          f[i] = two.x * unit[a];
          f[i + 1] = two.y * unit[a];
        }
        put(a, f);
      }
    } else {
      // 0 is a subnormal number, 255 NaN.  Of 2^126 and 2^127 a value may be past fp32 where its product with the row's
      // factor is not: a sixteenth of it has the same one rounding (the least such product is 2^-28).
#pragma unroll
      for (int a = 0; a < kAhead; ++a) {
        const bool far = s[a] - 253u < 2u;
        const float value = __uint_as_float(s[a] == 0u ? 0x00400000u : (s[a] == 255u ? 0x7FFFFFFFu : (s[a] - (far ? 4u : 0u)) << 23));
        const float back = far ? 16.0f : 1.0f;
        float f[V];
#pragma unroll
        for (int i = 0; i < V; i += 2) {
          const float2 two = pair_values((c[a] >> (4 * i)) & 255u);
          f[i] = two.x * value * by * back;
          f[i + 1] = two.y * value * by * back;
        }
        put(a, f);
      }
    }
  }
}

// Whether rows of a buffer start at multiples of `bytes` (a power of two).
bool rows_at(const void* p, int64_t ld_bytes, int64_t n, int bytes) {
  return ((reinterpret_cast<uintptr_t>(p) | (n > 1 ? (uintptr_t)ld_bytes : 0)) & (uintptr_t)(bytes - 1)) == 0;
}

unsigned grid_of(int64_t units, int per_cta) {
  return (unsigned)std::min<int64_t>((units + per_cta - 1) / per_cta, 64ll * sm_count());
}

// Four loads ahead where a row has as many and every SM a few dozen warps' units of them (8192 x 8192 bf16
// 34 us).
bool ahead_pays(int64_t n, int K, int V) { return K >= 128 * V && n * (K / (128 * V)) >= 32ll * sm_count(); }
template <typename T, int V, bool kWideX, bool kWideQ, int kAhead>
cudaError_t launch_units(const Mx4QuantArgs& A, cudaStream_t st) {
  const int64_t parts = ((int64_t)A.K + 32 * V * kAhead - 1) / (32 * V * kAhead);
  return launch_kernel(k_mx4_quantize<T, V, kWideX, kWideQ, kAhead>, dim3(grid_of(A.n * parts, kThreads / 32)), dim3(kThreads), 0, st,
                       true, A);
}
template <typename T, int V, bool kWideX, bool kWideQ>
cudaError_t launch_plain(const Mx4QuantArgs& A, cudaStream_t st) {
  return ahead_pays(A.n, A.K, V) ? launch_units<T, V, kWideX, kWideQ, 4>(A, st) : launch_units<T, V, kWideX, kWideQ, 1>(A, st);
}

template <typename T, bool kRes, bool kSmall, int V, bool kWide>
cudaError_t launch_norm(const Mx4QuantArgs& A, cudaStream_t st) {
  constexpr int kAhead = 2;
  const int64_t vecs = ((int64_t)A.K + V - 1) / V;
  if (vecs <= 128)
    return launch_kernel(k_mx4_norm<T, kRes, kSmall, V, kWide, kAhead, true>, dim3((unsigned)((A.n + kThreads / 32 - 1) / (kThreads / 32))),
                         dim3(kThreads), 0, st, true, A);
  // (few rows: a thread of its own for each vector, and none ahead; 1 x 8192 bf16 with residual)
  if (A.n <= 2 * sm_count() && vecs <= 1024)
    return launch_kernel(k_mx4_norm<T, kRes, kSmall, V, kWide, 1, false>, dim3((unsigned)A.n), dim3((unsigned)((vecs + 31) / 32 * 32)), 0, st,
                         true, A);
  const int64_t want = A.n <= 2 * sm_count() ? vecs : (vecs + kAhead - 1) / kAhead;
  // (many rows: small CTAs, of which an SM has room for many; with residual, 128, 256, 512 and 1024 threads:
  // 31,754 x 9856 bf16 315, 373, 484, 554 us, 8191 x 4096 36.6, 40.3, 40.4, 40.4; 3000 x 9857 fp32 77, 70, 80, 115)
  const int most = A.n <= 2 * sm_count() ? 1024 : (A.n < 4096 ? 256 : 128);
  const int threads = (int)std::min<int64_t>(most, (want + 31) / 32 * 32);
  return launch_kernel(k_mx4_norm<T, kRes, kSmall, V, kWide, kAhead, false>, dim3((unsigned)A.n), dim3((unsigned)threads), 0, st, true, A);
}

template <typename T, int V, bool kWide>
cudaError_t launch_rows(const Mx4QuantArgs& A, cudaStream_t st) {
  // (the squares of fp16 values do not leave fp32)
  if constexpr (!std::is_same<T, __half>::value)
    if (A.eps < kSmallEps) return A.res ? launch_norm<T, true, true, V, kWide>(A, st) : launch_norm<T, false, true, V, kWide>(A, st);
  return A.res ? launch_norm<T, true, false, V, kWide>(A, st) : launch_norm<T, false, false, V, kWide>(A, st);
}

template <typename T>
cudaError_t launch_type(const Mx4QuantArgs& A, bool norm, cudaStream_t st) {
  constexpr int V = 16 / (int)sizeof(T);
  constexpr int64_t kSize = (int64_t)sizeof(T);
  const bool x = rows_at(A.x, A.ldx * kSize, A.n, 16), q = rows_at(A.q, A.ldq, A.n, V / 2);
  if (!norm) {
    if (x) return q ? launch_plain<T, V, true, true>(A, st) : launch_plain<T, V, true, false>(A, st);
    // (one by one: 20,000 x 2002 bf16 40 us by eight, 44 by four; 30,000 x 100 6.9, 5.8)
    if (A.K >= 1024 || V == 4) return q ? launch_plain<T, V, false, true>(A, st) : launch_plain<T, V, false, false>(A, st);
    return rows_at(A.q, A.ldq, A.n, 2) ? launch_plain<T, 4, false, true>(A, st) : launch_plain<T, 4, false, false>(A, st);
  }
  const bool wide = x && q && (!A.res || rows_at(A.res, A.ldr * kSize, A.n, 16)) &&
                    (!A.sum || rows_at(A.sum, A.lds * kSize, A.n, 16)) && rows_at(A.gain, 0, 1, 16);
  // (of 16 bits too four values, whose loads and stores one by one are fewer at a time)
  return wide ? launch_rows<T, V, true>(A, st) : launch_rows<T, 4, false>(A, st);
}

template <typename T, int V, int kAhead>
cudaError_t launch_back(const Mx4DequantArgs& A, cudaStream_t st) {
  const int64_t parts = ((int64_t)A.K + 32 * V * kAhead - 1) / (32 * V * kAhead);
  return launch_kernel(k_mx4_dequantize<T, V, kAhead>, dim3(grid_of(A.n * parts, kThreads / 32)), dim3(kThreads), 0, st, true, A);
}
template <typename T, int V>
cudaError_t launch_back(const Mx4DequantArgs& A, cudaStream_t st) {
  return ahead_pays(A.n, A.K, V) ? launch_back<T, V, 4>(A, st) : launch_back<T, V, V == 2 ? 2 : 1>(A, st);
}
template <typename T>
cudaError_t launch_dequant(const Mx4DequantArgs& A, cudaStream_t st) {
  const bool wide = rows_at(A.out, A.ldo * (int64_t)sizeof(T), A.n, 16) && rows_at(A.q, A.ldq, A.n, 4);
  return wide ? launch_back<T, 8>(A, st) : launch_back<T, 2>(A, st);
}

}  // namespace

cudaError_t launch_mx4_quantize(const Mx4QuantArgs& A, bool norm, cudaStream_t st) {
  if (A.type == BMLP_F32) return launch_type<float>(A, norm, st);
  return A.type == BMLP_F16 ? launch_type<__half>(A, norm, st) : launch_type<__nv_bfloat16>(A, norm, st);
}

cudaError_t launch_mx4_dequantize(const Mx4DequantArgs& A, cudaStream_t st) {
  if (A.type == BMLP_F32) return launch_dequant<float>(A, st);
  return A.type == BMLP_F16 ? launch_dequant<__half>(A, st) : launch_dequant<__nv_bfloat16>(A, st);
}

}  // namespace bk
