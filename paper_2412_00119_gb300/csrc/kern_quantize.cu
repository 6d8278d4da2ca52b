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
// k_quantize_regs: a row's threads (a warp, or a CTA of up to 1,024) hold it in
// registers, so memory is read and written once.  Vectors of 16 bytes where the rows
// of every buffer allow them, else of 4 bytes or single values.  Bound: memory.
//
// k_quantize_long: rows too long for that, read twice.  Also rows of any length where eps
// does not hold up squares that leave fp32 (kSmallEps).
#include <algorithm>
#include <type_traits>

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

// Below this eps (2^-80) a row's scale may hang on squares that are lost in fp32, those of
// |h| < 2^-63.  Such rows have a sum below kSmallSum (2^-90: what a greater one has lost is
// less than 2^-60 of it for each value), every |h| below 2^-45, and squares of h kUp (2^85)
// that are inside fp32's range down to its least subnormal.
constexpr float kSmallEps = 8.27180613e-25f, kSmallSum = 8.07793566e-28f;
constexpr float kUpA = 4398046511104.0f, kUpB = 2.0f * kUpA, kUp = kUpA * kUpB;   // 2^42, 2^43

// The row's code factor and scale from the bits of A and (norm) its sum of squares; small: of
// squares of h kUp.
struct RowScale {
  float inv, scale;
};
__device__ __forceinline__ RowScale row_scale(uint32_t abits, float sumsq, int K, float eps, bool norm, bool small = false) {
  RowScale r = {0.0f, __uint_as_float(0x7FFFFFFFu)};
  if (abits >= kInfBits || (norm && !(sumsq < __uint_as_float(kInfBits)))) return r;
  const float A = __uint_as_float(abits);
  r.scale = 0.0f;
  if (A < kLeast) return r;
  r.inv = 127.0f / A;
  r.scale = A / 127.0f;
  if (norm) {
    const float rstd = 1.0f / sqrtf(__fadd_rn(sumsq / (float)K, small ? eps * kUp * kUp : eps));
    r.scale = small ? (r.scale * kUpA) * (rstd * kUpB) : __fmul_rn(r.scale, rstd);
  }
  return r;
}

// |a| against the maximum so far; NaN if either is.
__device__ __forceinline__ float max_nan(float m, float a) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(m), "f"(fabsf(a)));
  return r;
}

// A code in the low byte: rint by an addition that leaves a unit in the last place
// (|u inv| <= 127 (1 + 2^-22)).
__device__ __forceinline__ uint32_t code(float u, float inv) {
  return __float_as_uint(__fadd_rn(__fmul_rn(u, inv), 12582912.0f));   // 1.5 2^23
}

// Sum and maximum over a row's threads: the warp, or the CTA's warps (one barrier).
template <bool kWarpRow>
__device__ __forceinline__ void row_reduce(float& sq, uint32_t& most, bool norm, int turn) {
  if (norm) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sq += __shfl_xor_sync(kFullMask, sq, o);
  }
  most = __reduce_max_sync(kFullMask, most);
  if constexpr (!kWarpRow) {
    // rows alternate between two places: a warp may write the next row's while another
    // still reads this one's
    __shared__ float ssums[2][32];
    __shared__ uint32_t smaxs[2][32];
    float* ssum = ssums[turn & 1];
    uint32_t* smax = smaxs[turn & 1];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    if (lane == 0) {
      ssum[warp] = sq;
      smax[warp] = most;
    }
    __syncthreads();
    sq = lane < warps ? ssum[lane] : 0.0f;
    most = lane < warps ? smax[lane] : 0u;
    if (norm) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) sq += __shfl_xor_sync(kFullMask, sq, o);
    }
    most = __reduce_max_sync(kFullMask, most);
  }
}

// V values as they lie in memory.
template <typename T, int V> struct Pack {
  static constexpr int kBytes = V * (int)sizeof(T);
  uint32_t w[(kBytes + 3) / 4];
  // values [skip, left) of those from p on, which are the row's; zeros in the others' place
  // (kWhole: all or none are)
  template <bool kWhole>
  __device__ __forceinline__ void load(const T* p, int skip, int left) {
#pragma unroll
    for (int i = 0; i < (kBytes + 3) / 4; ++i) w[i] = 0u;
    if (skip <= 0 && left >= V) {
      if constexpr (kBytes == 16) {
        const uint4 v = *reinterpret_cast<const uint4*>(p);
        w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
      } else if constexpr (kBytes == 4) {
        w[0] = *reinterpret_cast<const uint32_t*>(p);
      } else {
        w[0] = *reinterpret_cast<const uint16_t*>(p);
      }
    } else if constexpr (V > 1 && !kWhole) {
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (i >= skip && i < left) {
          if constexpr (sizeof(T) == 4) w[i] = *reinterpret_cast<const uint32_t*>(p + i);
          else w[i / 2] |= (uint32_t)*reinterpret_cast<const uint16_t*>(p + i) << (16 * (i % 2));
        }
    }
  }
  template <bool kWhole>
  __device__ __forceinline__ void store(T* p, int skip, int left) const {
    if (skip <= 0 && left >= V) {
      if constexpr (kBytes == 16) *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
      else if constexpr (kBytes == 4) *reinterpret_cast<uint32_t*>(p) = w[0];
      else *reinterpret_cast<uint16_t*>(p) = (uint16_t)w[0];
    } else if constexpr (V > 1 && !kWhole) {
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (i >= skip && i < left) {
          if constexpr (sizeof(T) == 4) *reinterpret_cast<uint32_t*>(p + i) = w[i];
          else *reinterpret_cast<uint16_t*>(p + i) = (uint16_t)(w[i / 2] >> (16 * (i % 2)));
        }
    }
  }
  __device__ __forceinline__ float get(int i) const {
    if constexpr (std::is_same<T, float>::value) return __uint_as_float(w[i]);
    else if constexpr (std::is_same<T, __half>::value) return __half2float(__ushort_as_half((unsigned short)(w[i / 2] >> (16 * (i % 2)))));
    else return __uint_as_float(i % 2 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
  }
  __device__ __forceinline__ void set(const float (&f)[V]) {
    if constexpr (std::is_same<T, float>::value) {
#pragma unroll
      for (int i = 0; i < V; ++i) w[i] = __float_as_uint(f[i]);
    } else {
#pragma unroll
      for (int i = 0; i < V; i += 2) {
        const T a = from_f32<T>(f[i]), b = from_f32<T>(i + 1 < V ? f[i + 1] : 0.0f);
        w[i / 2] = (uint32_t)*reinterpret_cast<const uint16_t*>(&a) | (uint32_t)*reinterpret_cast<const uint16_t*>(&b) << 16;
      }
    }
  }
};

template <int V>
__device__ __forceinline__ void make_codes(uint32_t (&w)[(V + 3) / 4], const float (&u)[V], float inv, uint32_t live) {
#pragma unroll
  for (int i = 0; i < (V + 3) / 4; ++i) {
    uint32_t c[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) c[e] = 4 * i + e < V ? code(u[4 * i + e < V ? 4 * i + e : 0], inv) : 0u;
    const uint32_t lo = V > 1 ? __byte_perm(c[0], c[1], 0x0040) : c[0];
    w[i] = (V > 2 ? __byte_perm(lo, __byte_perm(c[2], c[3], 0x0040), 0x5410) : lo) & live;
  }
}

// p aligned to V codes.
template <int V, bool kWhole>
__device__ __forceinline__ void store_codes(int8_t* p, const uint32_t (&w)[(V + 3) / 4], int left) {
  if (left >= V) {
    if constexpr (V == 8) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    else if constexpr (V == 4) *reinterpret_cast<uint32_t*>(p) = w[0];
    else if constexpr (V == 2) *reinterpret_cast<uint16_t*>(p) = (uint16_t)w[0];
    else *p = (int8_t)w[0];
  } else if constexpr (V > 1 && !kWhole) {
#pragma unroll
    for (int i = 0; i < V - 1; ++i)
      if (i < left) p[i] = (int8_t)(w[i / 4] >> (8 * (i % 4)));
  }
}

// `count` values of a row (U: their bits) from shared memory, where value e begins at byte e sizeof(U) + apart of buf
// (16-byte aligned, 16 bytes before it and after its last), to `to`, anywhere: a thread of
// `threads` takes aligned 16 bytes of it at a time.
template <typename U>
__device__ __forceinline__ void copy_row(U* to, const uint8_t* buf, int apart, int count, int tid, int threads) {
  constexpr int kEach = 16 / (int)sizeof(U);
  const int before = (int)(reinterpret_cast<uintptr_t>(to) & 15) / (int)sizeof(U);
  for (int e = kEach * tid - before; e < count; e += kEach * threads) {
    const int at = e * (int)sizeof(U) + apart;            // (from -15 on)
    const uint32_t* w = reinterpret_cast<const uint32_t*>(buf + (at & ~3));
    uint32_t v[4];
    uint32_t x = w[0];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t y = w[i + 1];
      v[i] = __funnelshift_r(x, y, 8u * (uint32_t)(at & 3));
      x = y;
    }
    if (e >= 0 && e + kEach <= count) {
      *reinterpret_cast<uint4*>(to + e) = make_uint4(v[0], v[1], v[2], v[3]);
    } else {
#pragma unroll
      for (int i = 0; i < kEach; ++i)
        if (e + i >= 0 && e + i < count) to[e + i] = (U)(v[i * (int)sizeof(U) / 4] >> (8 * (i * (int)sizeof(U) % 4)));
    }
  }
}

constexpr int kRowsPerCta = 8;   // rows of a CTA with a warp each
// What is done to a row (residual: its registers are there only where it is).
constexpr int kPlain = 0, kNormed = 1, kResidual = 2;

// Shared memory of a row's codes, or of its sums: a vector per thread and turn, 16 bytes before
// and after.
__host__ __device__ constexpr int row_bytes(int nv, int threads, int vector) { return nv * threads * vector + 32; }

// CTAs that an SM holds at least, by the registers each may have, where a warp's norm of a row has
// 32 values per lane (us; without a bound the compiler takes more than help): 60,000 x 784 fp32 38
// with four, 41 without; with residual 65,536 x 784 bf16 59 with three, 69; rows at odd places
// 60,000 x 785 bf16 57 with two, 70 with three, 93, but 60,000 x 1001 fp32
// with residual 125 without, 137 with two.
template <typename T, int kMode, int kValues, bool kWarpRow, bool kWhole>
__host__ __device__ constexpr int least_ctas() {
  if (!kWarpRow || kValues <= 16 || kMode == kPlain) return 1;
  if (!kWhole) return kMode == kResidual && sizeof(T) == 4 ? 1 : 2;
  return kMode == kNormed ? 4 : 3;
}

// A row's T threads hold it: vector v of thread t is v T + t, NV vectors of V values
// each.  The grid walks the rows; a row's values are loaded while the row before is
// reduced and written, and the gain stays in registers (kAhead; without it neither,
// where the registers do not hold both).
// kApart: rows that do not start at multiples of 16 bytes, the inputs' equally far from one.
// A thread's vectors are the aligned 16 bytes around the row; rows eight apart lie
// alike, and a thread's rows are a multiple of eight apart.  The codes go through shared
// memory, since theirs lie otherwise, and the sums where theirs do (apart_sum).
// kWhole: K is a multiple of V, and no vector is partly the row's.
template <typename T, int kMode, int V, int NV, bool kWarpRow, bool kAhead, bool kApart, bool kWhole>
__global__ void __launch_bounds__(kWarpRow ? 32 * kRowsPerCta : 1024, (least_ctas<T, kMode, V * NV, kWarpRow, kWhole>()))
    k_quantize_regs(const QuantArgs A, bool apart_sum) {
  pdl_wait();
  pdl_trigger();
  const int threads = kWarpRow ? 32 : (int)blockDim.x;
  const int tid = kWarpRow ? (int)(threadIdx.x & 31) : (int)threadIdx.x;
  const int64_t step = kWarpRow ? (int64_t)gridDim.x * kRowsPerCta : (int64_t)gridDim.x;
  int64_t row = kWarpRow ? (int64_t)blockIdx.x * kRowsPerCta + (threadIdx.x >> 5) : (int64_t)blockIdx.x;
  const T* x = static_cast<const T*>(A.x);
  constexpr bool kNorm = kMode != kPlain, kRes = kMode == kResidual;
  const T* res = static_cast<const T*>(A.res);
  T* sum = kNorm ? static_cast<T*>(A.sum) : nullptr;
  const T* gain = kNorm ? static_cast<const T*>(A.gain) : nullptr;
  extern __shared__ uint4 smem_codes[];
  uint8_t* codes = reinterpret_cast<uint8_t*>(smem_codes) + 16 + (kWarpRow ? (int)(threadIdx.x >> 5) * row_bytes(NV, 32, V) : 0);
  uint8_t* sums = reinterpret_cast<uint8_t*>(smem_codes) + 16 + (kWarpRow ? kRowsPerCta : 1) * row_bytes(NV, threads, V) +
                  (kWarpRow ? (int)(threadIdx.x >> 5) * row_bytes(NV, 32, 16) : 0);
  const int apart = kApart ? (int)((reinterpret_cast<uintptr_t>(x + row * A.ldx) & 15) / sizeof(T)) : 0;
  auto at = [&](int v) { return (v * threads + tid) * V - apart; };
  auto skip = [&](int v) { return kApart ? -at(v) : 0; };
  Pack<T, V> px[NV], pr[kRes ? NV : 1], pg[kAhead ? NV : 1];
  auto load_gain = [&](int v, Pack<T, V>& to) {
    if constexpr (kApart) {
      // (the gain lies otherwise than the rows: value by value)
#pragma unroll
      for (int i = 0; i < (Pack<T, V>::kBytes + 3) / 4; ++i) to.w[i] = 0u;
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (at(v) + i >= 0 && at(v) + i < A.K) {
          if constexpr (sizeof(T) == 4) to.w[i] = reinterpret_cast<const uint32_t*>(gain)[at(v) + i];
          else to.w[i / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(gain)[at(v) + i] << (16 * (i % 2));
        }
    } else {
      to.template load<kWhole>(gain + at(v), 0, A.K - at(v));
    }
  };
  if (kAhead && gain && row < A.n) {
#pragma unroll
    for (int v = 0; v < NV; ++v) load_gain(v, pg[kAhead ? v : 0]);
  }
  auto load = [&](int64_t i) {
#pragma unroll
    for (int v = 0; v < NV; ++v) px[v].template load<kWhole>(x + i * A.ldx + at(v), skip(v), A.K - at(v));
    if constexpr (kRes) {
#pragma unroll
      for (int v = 0; v < NV; ++v) pr[v].template load<kWhole>(res + i * A.ldr + at(v), skip(v), A.K - at(v));
    }
  };
  if (kAhead && row < A.n) load(row);
  for (int turn = 0; row < A.n; row += step, turn ^= 1) {
    if (!kAhead) load(row);
    float u[NV][V];
    float sq = 0.0f, most = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        u[v][i] = px[v].get(i);
        if constexpr (kRes) u[v][i] = __fadd_rn(u[v][i], pr[v].get(i));
      }
    // (this row is read: sum_out may be x or res)
    if (kAhead && row + step < A.n) load(row + step);
    if (sum) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        Pack<T, V> ps;
        ps.set(u[v]);
        // (the row before was copied from there before its codes were)
        if constexpr (kApart) {
          if (apart_sum) *reinterpret_cast<uint4*>(sums + 16 * (v * threads + tid)) = make_uint4(ps.w[0], ps.w[1], ps.w[2], ps.w[3]);
        }
        if (!kApart || !apart_sum) ps.template store<kWhole>(sum + row * A.lds + at(v), skip(v), A.K - at(v));
      }
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      if (!kAhead && gain) load_gain(v, pg[0]);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        if (kNorm) sq += u[v][i] * u[v][i];
        if (gain) u[v][i] = __fmul_rn(u[v][i], pg[kAhead ? v : 0].get(i));
        most = max_nan(most, u[v][i]);
      }
    }
    uint32_t mbits = __float_as_uint(most);
    row_reduce<kWarpRow>(sq, mbits, kNorm, turn);
    if (kApart && apart_sum) {   // (only where there are sums)
      if constexpr (kWarpRow) __syncwarp();   // (a CTA's threads have met in row_reduce)
      using Bits = std::conditional_t<sizeof(T) == 4, uint32_t, uint16_t>;
      copy_row(reinterpret_cast<Bits*>(sum + row * A.lds), sums, apart * (int)sizeof(T), A.K, tid, threads);
    }
    const RowScale r = row_scale(mbits, sq, A.K, A.eps, kNorm);
    const uint32_t live = r.inv == 0.0f ? 0u : 0xFFFFFFFFu;
    int8_t* q = A.q + row * A.ldq;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      uint32_t w[(V + 3) / 4];
      make_codes<V>(w, u[v], r.inv, live);
      if constexpr (!kApart) {
        store_codes<V, kWhole>(q + at(v), w, A.K - at(v));
      } else {
        // (the row before was copied from there by threads that have since met in row_reduce)
        uint8_t* to = codes + (v * threads + tid) * V;
        if constexpr (V == 8) *reinterpret_cast<uint2*>(to) = make_uint2(w[0], w[(V + 3) / 4 - 1]);
        else *reinterpret_cast<uint32_t*>(to) = w[0];
      }
    }
    if constexpr (kApart) {
      if constexpr (kWarpRow) __syncwarp();
      else __syncthreads();
      copy_row(q, codes, apart, A.K, tid, threads);
      if constexpr (kWarpRow) __syncwarp();
    }
    if (tid == 0) A.scale[row] = r.scale;
  }
}

constexpr int kThreads = 1024;

// A CTA per row; a warp where rows are short (only with kSmall: 60,000 x 784 fp32 83 us, by CTAs 574;
// in registers, at other eps, 38.  The two sums there cost every call 6%, at any eps).
// kSmall: eps < kSmallEps.
template <typename T, int kMode, bool kSmall, bool kWarpRow>
__global__ void __launch_bounds__(kThreads) k_quantize_long(const QuantArgs A) {
  constexpr bool kNorm = kMode != kPlain;
  constexpr uint32_t kStep = kWarpRow ? 32 : kThreads;
  pdl_wait();
  pdl_trigger();
  const T* gain = static_cast<const T*>(A.gain);
  const uint32_t tid = threadIdx.x % kStep;
  const int64_t row = kWarpRow ? (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5) : (int64_t)blockIdx.x;
  if (kWarpRow && row >= A.n) return;
  const T* x = static_cast<const T*>(A.x) + row * A.ldx;
  const T* res = kNorm && A.res ? static_cast<const T*>(A.res) + row * A.ldr : nullptr;
  T* sum = kNorm && A.sum ? static_cast<T*>(A.sum) + row * A.lds : nullptr;
  auto h_of = [&](uint32_t i) { return res ? __fadd_rn(to_f32(x[i]), to_f32(res[i])) : to_f32(x[i]); };
  auto u_of = [&](float h, uint32_t i) { return kNorm && gain ? __fmul_rn(h, to_f32(gain[i])) : h; };
  float sq = 0.0f, sq_up = 0.0f, most = 0.0f;
  for (uint32_t i = tid; i < (uint32_t)A.K; i += kStep) {
    const float h = h_of(i);
    sq += h * h;
    if (kSmall) sq_up += (h * kUp) * (h * kUp);
    most = max_nan(most, u_of(h, i));
  }
  uint32_t mbits = __float_as_uint(most);
  row_reduce<kWarpRow>(sq, mbits, kNorm, 0);
  const bool small = kSmall && sq < kSmallSum;
  if (kSmall) row_reduce<kWarpRow>(sq_up, mbits, kNorm, 1);
  const RowScale r = row_scale(mbits, small ? sq_up : sq, A.K, A.eps, kNorm, small);
  const uint32_t live = r.inv == 0.0f ? 0u : 0xFFFFFFFFu;
  // the row's values again: a thread writes its own elements of sum_out only after
  // it has read them (sum_out may be x or res)
  for (uint32_t i = tid; i < (uint32_t)A.K; i += kStep) {
    const float h = h_of(i);
    if (sum) sum[i] = from_f32<T>(h);
    A.q[row * A.ldq + i] = (int8_t)(code(u_of(h, i), r.inv) & live);
  }
  if (tid == 0) A.scale[row] = r.scale;
}

// A warp per row.  With 32 values per lane whole rows run faster from more warps than with the next
// row loaded ahead (65,536 x 784 bf16 31 us, ahead 40; 60,000 x 784 fp32 38, ahead 55;
// 60,000 x 1000 bf16 coded 28.6, ahead 32.5), rows with a ragged end in 16 bits or at odd places not.
template <typename T, int kMode, int V, int NV, bool kApart, bool kWhole>
cudaError_t launch_warp_rows(const QuantArgs& A, bool apart_sum, cudaStream_t st) {
    constexpr bool kAhead = V * NV <= 16 || (sizeof(T) == 2 && kMode != kPlain && !kWhole) || kApart;
  const int64_t ctas = std::min((A.n + kRowsPerCta - 1) / kRowsPerCta, (int64_t)(kAhead && V * NV > 16 ? 4 : 8) * sm_count());
  return launch_kernel(k_quantize_regs<T, kMode, V, NV, true, kAhead, kApart, kWhole>, dim3((unsigned)ctas), dim3(32 * kRowsPerCta),
                       kApart ? (size_t)kRowsPerCta * (row_bytes(NV, 32, V) + (apart_sum ? row_bytes(NV, 32, 16) : 0)) : 0, st, true,
                       A, apart_sum);
}

// A CTA per row: 1,024 threads an SM.
template <typename T, int kMode, int V, int NV, bool kApart, bool kWhole>
cudaError_t launch_cta_rows(const QuantArgs& A, bool apart_sum, cudaStream_t st) {
  const int vecs = kApart ? (int)((A.K + 2ll * V - 2) / V) : A.K / V + (A.K % V != 0);
  const int threads = (vecs + 32 * NV - 1) / (32 * NV) * 32;
  constexpr bool kAhead = !(kMode != kPlain && V * NV > (sizeof(T) == 2 ? 16 : 8));
  const int64_t ctas = kAhead ? std::min(A.n, (int64_t)(1024 / threads) * sm_count() / 8 * 8) : A.n;
  if (kApart && apart_sum) {
    static std::atomic<uint64_t> done{0};
    const cudaError_t e = allow_smem(done, k_quantize_regs<T, kMode, V, NV, false, kAhead, kApart, kWhole>,
                                     row_bytes(NV, 1024, V) + row_bytes(NV, 1024, 16));
    if (e != cudaSuccess) return e;
  }
  return launch_kernel(k_quantize_regs<T, kMode, V, NV, false, kAhead, kApart, kWhole>, dim3((unsigned)ctas), dim3((unsigned)threads),
                       kApart ? (size_t)row_bytes(NV, threads, V) + (apart_sum ? row_bytes(NV, threads, 16) : 0) : 0, st, true, A,
                       apart_sum);
}

// Which form (us, rows in bf16 unless said): rows that a warp holds in at most kWarpMost
// vectors per lane get a warp each (65,536 x 784 31, by CTAs 58; 60,000 x 784 fp32 38, by CTAs
// 62).  Else a CTA per row, with one vector per thread for few rows (1 x 8192 2.5, two 2.8, four 4.1), and
// for many as many as the registers hold beside the next row's: four without a norm
// (8192 x 8192 30, two 34, one 44), two with it (8191 x 4096 with residual 40, four 57 for want of registers).
template <typename T, int kMode, int V, bool kApart, bool kWhole>
cudaError_t launch_v(const QuantArgs& A, bool apart_sum, cudaStream_t st) {
  constexpr int kWarpMost = V == 8 ? 4 : (V == 4 ? 8 : 16);
  const int64_t vecs = kApart ? (A.K + 2ll * V - 2) / V : A.K / V + (A.K % V != 0);
  if constexpr (!kApart) {
    if (vecs <= 32) return launch_warp_rows<T, kMode, V, 1, false, kWhole>(A, apart_sum, st);
    if (vecs <= 64) return launch_warp_rows<T, kMode, V, 2, false, kWhole>(A, apart_sum, st);
    if (vecs <= 128) return launch_warp_rows<T, kMode, V, 4, false, kWhole>(A, apart_sum, st);
    if (V <= 2 && vecs <= 256) return launch_warp_rows<T, kMode, V, V <= 2 ? 8 : 4, false, kWhole>(A, apart_sum, st);
  }
  if (vecs <= 32 * kWarpMost) return launch_warp_rows<T, kMode, V, kWarpMost, kApart, kWhole>(A, apart_sum, st);
  if (vecs > 4096)
    return launch_kernel(k_quantize_long<T, kMode, false, false>, dim3((unsigned)A.n), dim3(kThreads), 0, st, true, A);
  const bool few = A.n <= 2 * sm_count();
  if (vecs > 2048 || (!few && (V <= 2 || kMode == kPlain))) return launch_cta_rows<T, kMode, V, 4, kApart, kWhole>(A, apart_sum, st);
  if (vecs > 1024 || !few) return launch_cta_rows<T, kMode, V, 2, kApart, kWhole>(A, apart_sum, st);
  return launch_cta_rows<T, kMode, V, 1, kApart, kWhole>(A, apart_sum, st);
}

// Vectors of 16 bytes; also where rows start elsewhere but the inputs' alike, if they are long and
// many (us, by single values after it: 8191 x 4095 bf16 with residual 68, 98; 60,000 x 1001 bf16
// coded 51, 66; but 60,000 x 255 25, 13, and 100 x 1001 4.3, 2.1) or too long for single values;
// else of 4 bytes or single values.
template <typename T, int kMode>
cudaError_t launch_type(const QuantArgs& A, cudaStream_t st) {
  constexpr int V = 16 / (int)sizeof(T);
  // (the squares of fp16 values do not leave fp32)
  if constexpr (kMode != kPlain && !std::is_same<T, __half>::value)
    if (A.eps < kSmallEps) {
      constexpr int kEach = kThreads / 32;
      if (A.K > 2048) return launch_kernel(k_quantize_long<T, kMode, true, false>, dim3((unsigned)A.n), dim3(kThreads), 0, st, true, A);
      return launch_kernel(k_quantize_long<T, kMode, true, true>, dim3((unsigned)((A.n + kEach - 1) / kEach)), dim3(kThreads), 0, st,
                           true, A);
    }
  const bool many = A.n > 1;
  auto place = [&](const void* p, int64_t ld) {   // of a buffer's first rows, in 16 bytes
    return (reinterpret_cast<uintptr_t>(p) & 15) | (many ? (uintptr_t)(ld * (int64_t)sizeof(T)) & 15 : 0) << 4;
  };
  const uintptr_t px = place(A.x, A.ldx);
  const uintptr_t wide = px | (A.res ? place(A.res, A.ldr) : 0) | (A.sum ? place(A.sum, A.lds) : 0) |
                         (reinterpret_cast<uintptr_t>(A.gain) & 15);
  const uintptr_t codes = reinterpret_cast<uintptr_t>(A.q) | (many ? (uintptr_t)A.ldq : 0);
  if (wide == 0 && codes % V == 0)
    return A.K % V ? launch_v<T, kMode, V, false, false>(A, false, st) : launch_v<T, kMode, V, false, true>(A, false, st);
  const bool apart_sum = A.sum && place(A.sum, A.lds) != px;
  if ((!A.res || place(A.res, A.ldr) == px) && A.K > 512 && (A.n > 2 * sm_count() || A.K > 4096) && A.K <= 2048 * V - V)
    return launch_v<T, kMode, V, true, false>(A, apart_sum, st);
  if (sizeof(T) == 2 && (wide & 0x33) == 0 && codes % 2 == 0) return launch_v<T, kMode, sizeof(T) == 2 ? 2 : 1, false, false>(A, false, st);
  return launch_v<T, kMode, 1, false, false>(A, false, st);
}

template <typename T>
cudaError_t launch_any(const QuantArgs& A, bool norm, cudaStream_t st) {
  return !norm ? launch_type<T, kPlain>(A, st) : (A.res ? launch_type<T, kResidual>(A, st) : launch_type<T, kNormed>(A, st));
}

}  // namespace

cudaError_t launch_quantize(const QuantArgs& all, bool norm, cudaStream_t st) {
  constexpr int64_t kMaxRows = 1ll << 30;   // of a launch
  const int64_t size = all.type == BMLP_F32 ? 4 : 2;
  for (int64_t off = 0; off < all.n; off += kMaxRows) {
    QuantArgs A = all;
    A.n = all.n - off < kMaxRows ? all.n - off : kMaxRows;
    A.x = static_cast<const uint8_t*>(all.x) + off * all.ldx * size;
    if (all.res) A.res = static_cast<const uint8_t*>(all.res) + off * all.ldr * size;
    if (all.sum) A.sum = static_cast<uint8_t*>(all.sum) + off * all.lds * size;
    A.q += off * all.ldq;
    A.scale += off;
    const cudaError_t e = all.type == BMLP_F32 ? launch_any<float>(A, norm, st)
                          : all.type == BMLP_F16 ? launch_any<__half>(A, norm, st)
                                                 : launch_any<__nv_bfloat16>(A, norm, st);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace bk
