// mx4_common.cuh -- what the kernels of the microscaled 4-bit product share: maps of the operands, the groups'
// row tiles, outputs, waits, the scales' way to shared memory, and sums on CUDA cores.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "int8_common.cuh"
#include "tc_common.cuh"

namespace bk {
namespace mx4 {

// Map of rows of codes, 128 bytes of box_rows rows at a time, in the 128B-swizzled order that the MMAs read;
// groups > 0: of groups of rows.  (Rows and groups start at multiples of 16 bytes.)
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
  if (!encode) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)bytes, (cuuint64_t)rows, (cuuint64_t)groups};
  const cuuint64_t strides[2] = {(cuuint64_t)ld, (cuuint64_t)group_ld};
  const cuuint32_t box[3] = {128, (cuuint32_t)box_rows, 1}, steps[3] = {1, 1, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, groups > 0 ? 3 : 2, const_cast<uint8_t*>(codes), dims, strides, box, steps,
                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// Maps of a call's codes: of the channels (128 at a time) and of the rows.
struct Maps {
  CUtensorMap w, a;
};

// Whether tensor copies can take the codes of both.
inline bool codes_whole(const Mx4Args& A) {
  const uint64_t a = A.n > 1 ? (uint64_t)A.lda : 0, w = A.N > 1 ? (uint64_t)A.ldw : 0, g = A.E > 1 ? (uint64_t)A.gw : 16;
  return ((reinterpret_cast<uintptr_t>(A.a) | reinterpret_cast<uintptr_t>(A.w) | a | w | g) & 15) == 0 && g != 0 &&
         a < (1ull << 40) && w < (1ull << 40) && g < (1ull << 40);
}
// Whether every row's scales start at a multiple of 16 bytes.
inline bool scales_whole(const Mx4Args& A) {
  return ((reinterpret_cast<uintptr_t>(A.as) | reinterpret_cast<uintptr_t>(A.ws) | (uintptr_t)(A.n > 1 ? A.ldas : 0) |
           (uintptr_t)(A.N > 1 ? A.ldws : 0) | (uintptr_t)(A.E > 1 ? A.gws : 0)) & 15) == 0;
}

// Rows [first, last) of a group.  Offsets that decrease or leave 0..n are taken as the
// nearest that do not: callers pass the largest offset before as `low`.
__device__ __forceinline__ int clamp_offset(int32_t offset, int low, int64_t n) {
  return max(low, min((int)n, (int)offset));
}

using i8::out_cast;

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

// An output from its sum; rs 1, bias 0 where there is none.
template <typename T>
__device__ __forceinline__ T output(float sum, float rs, float bias) { return out_cast<T>(__fadd_rn(__fmul_rn(sum, rs), bias)); }

// A lane's channel of 16 rows, of which `rows` are some: to[0], to[ldo], ..  rs: of row x in lane x.
template <typename T>
__device__ __forceinline__ void put_rows(T* to, int64_t ldo, const uint32_t (&sums)[16], float rs, float bias, int rows,
                                         bool live) {
  T y[16];
#pragma unroll
  for (int x = 0; x < 16; ++x) y[x] = output<T>(__uint_as_float(sums[x]), __shfl_sync(0xffffffffu, rs, x), bias);
  if (!live) return;
  if (rows >= 16) {
#pragma unroll
    for (int x = 0; x < 16; ++x, to += ldo) *to = y[x];
  } else {
#pragma unroll
    for (int x = 0; x < 15; ++x, to += ldo)
      if (x < rows) *to = y[x];
  }
}

// Bounded waits as in tc_common.cuh.  kPeer: with cluster-scope acquire (the barrier collects arrivals of the
// peer); kOrder: for arrivals that tell of tensor memory alone, which tcgen05's fences order around them.  A try may
// sleep for some 50 us, in place of many tries (16384 x 8192 -> 8192 by tiles 502 -> 498 us).
enum Wait { kHere, kPeer, kOrder };
template <Wait kWait = kHere>
__device__ __forceinline__ bool wait_phase(unsigned long long* bar, uint32_t parity, volatile int* failed,
                                           unsigned long long limit = tc::kWaitCycles) {
  const uint32_t a = tc::smem_u32(bar);
  uint32_t ok;
  auto try_wait = [&]() {
    if constexpr (kWait == kPeer)
      asm volatile(
          "{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2, 50000;\n"
          " selp.u32 %0, 1, 0, p;\n}"
          : "=r"(ok) : "r"(a), "r"(parity) : "memory");
    else if constexpr (kWait == kOrder)
      asm volatile(
          "{\n .reg .pred p;\n mbarrier.try_wait.parity.relaxed.cluster.shared::cta.b64 p, [%1], %2, 50000;\n"
          " selp.u32 %0, 1, 0, p;\n}"
          : "=r"(ok) : "r"(a), "r"(parity) : "memory");
    else
      asm volatile(
          "{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, 50000;\n"
          " selp.u32 %0, 1, 0, p;\n}"
          : "=r"(ok) : "r"(a), "r"(parity) : "memory");
  };
  try_wait();
  if (ok) return true;
  const unsigned long long t0 = clock64();
  while (true) {
    try_wait();
    if (ok) return true;
    if (*failed) return false;
    if (clock64() - t0 > limit) {
      *failed = 1;
      return false;
    }
  }
}

// Where a tile is.
struct Item {
  int e;          // group
  int rows;
  int64_t r0;     // first row
  int j0;         // first channel
};
// The row tiles of a call.
struct Items {
  const int32_t* tile0;   // by group: its first row tile (E + 1); null: one group
  const int32_t* row0;    // and its first row
  int E, nt, ctiles, step_u, step_c;
  int64_t rtiles, n;
  __device__ __forceinline__ Item at(int64_t u, int j0) const {
    Item it;
    it.j0 = j0;
    int64_t end = n;
    if (tile0) {
      int lo = 0, hi = E;      // the last group with tile0 <= u
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (tile0[mid] <= u) lo = mid; else hi = mid;
      }
      it.e = lo;
      it.r0 = row0[lo] + (u - tile0[lo]) * nt;
      end = row0[lo + 1];
    } else {
      it.e = 0;
      it.r0 = u * nt;
    }
    it.rows = (int)min((int64_t)nt, end - it.r0);
    return it;
  }
};
// The groups' first row tiles (groups[0..E]) and first rows (groups[E + 1..2 E + 1]), by one warp.
__device__ __forceinline__ void group_tiles(const Mx4Args& A, int nt, int32_t* groups) {
  const int lane = threadIdx.x & 31;
  int row = 0, tile = 0;
  for (int e0 = 0; e0 <= A.E; e0 += 32) {
    const int e = e0 + lane;
    int r = e <= A.E ? clamp_offset(A.offsets[e], 0, A.n) : 0;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
      const int v = __shfl_up_sync(0xffffffffu, r, o);
      if (lane >= o) r = max(r, v);
    }
    r = max(r, row);
    if (e <= A.E) groups[A.E + 1 + e] = r;
    row = __shfl_sync(0xffffffffu, r, 31);
  }
  __syncwarp();
  for (int e0 = 0; e0 <= A.E; e0 += 32) {
    const int e = e0 + lane;
    const int mine = e < A.E ? (groups[A.E + 2 + e] - groups[A.E + 1 + e] + nt - 1) / nt : 0;
    int t = mine;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
      const int v = __shfl_up_sync(0xffffffffu, t, o);
      if (lane >= o) t += v;
    }
    if (e <= A.E) groups[e] = tile + t - mine;
    tile += __shfl_sync(0xffffffffu, t, 31);
  }
}

// 128 channels' outputs of a tile on CUDA cores (rows first, first + step, ..), by all threads: only after a
// wait has expired.
static __device__ __noinline__ void plain_rows(const Mx4Args& A, const Item& it, int first, int step) {
  for (int64_t k = threadIdx.x; k < (int64_t)128 * it.rows; k += blockDim.x) {
    const int j = it.j0 + (int)(k % 128), x = (int)(k / 128);
    if (x % step == first && j < A.N) put_out(A, it.r0 + x, j, it.e, plain_sum(A, it.r0 + x, j, it.e));
  }
}

constexpr int kCell = 512;               // bytes of the scales of 128 rows x 128 codes: those of row r at 16 (r % 32) + 4 (r / 32)
// Descriptor of a cell: 32 rows of 16 bytes one after another, no swizzle.
__device__ __forceinline__ uint64_t cell_desc(uint32_t saddr) {
  uint64_t d = (saddr & 0x3FFFFu) >> 4;
  d |= (uint64_t)(128 >> 4) << 16;   // from 8 rows to the next, in either sense
  d |= (uint64_t)(128 >> 4) << 32;
  d |= (uint64_t)1 << 46;            // descriptor version (sm_100 family)
  return d;
}
__device__ __forceinline__ void sts32(uint32_t a, uint32_t v) {
  asm volatile("st.shared.u32 [%0], %1;" ::"r"(a), "r"(v) : "memory");
}

// kChunks aligned 16-byte chunks from p on, of which the first `size` bytes are read (none where size <= 0) and the
// rest are zeros; tail: where there may be a chunk of which a part is.  No branches: all loads are
// under way together.
template <int kChunks>
__device__ __forceinline__ void load_chunks(uint32_t (&v)[kChunks][4], const int8_t* p, int size, bool tail) {
#pragma unroll
  for (int h = 0; h < kChunks; ++h) {
    v[h][0] = v[h][1] = v[h][2] = v[h][3] = 0u;
    asm volatile("{\n .reg .pred q;\n setp.ge.s32 q, %5, 16;\n @q ld.global.nc.v4.u32 {%0, %1, %2, %3}, [%4];\n}"
                 : "+r"(v[h][0]), "+r"(v[h][1]), "+r"(v[h][2]), "+r"(v[h][3]) : "l"(p + 16 * h), "r"(size - 16 * h));
  }
  if (tail) {
    const int h = size >> 4, left = size > 0 && h < kChunks ? size & 15 : 0;   // the chunk, and its bytes
    uint32_t b[15];
#pragma unroll
    for (int x = 0; x < 15; ++x) {
      b[x] = 0u;
      asm volatile("{\n .reg .pred q;\n setp.gt.s32 q, %2, %3;\n @q ld.global.nc.u8 %0, [%1];\n}"
                   : "+r"(b[x]) : "l"(p + 16 * h + x), "r"(left), "r"(x));
    }
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      const uint32_t w = b[4 * y] | b[4 * y + 1] << 8 | b[4 * y + 2] << 16 | (y < 3 ? b[y < 3 ? 4 * y + 3 : 0] << 24 : 0u);
#pragma unroll
      for (int i = 0; i < kChunks; ++i)
        if (i == h) v[i][y] |= w;
    }
  }
}

// The scale bytes of 1024 codes (32) of a row from byte k (a multiple of 16) on, zeros from len on.  whole: every
// row starts at a multiple of 16 bytes.
__device__ __forceinline__ void load_scales(uint32_t (&v)[2][4], const uint8_t* row, bool live, bool whole, int k, int len) {
  const int8_t* p = reinterpret_cast<const int8_t*>(row);
  if (whole) {
    load_chunks<2>(v, p + k, live ? len - k : 0, len - k < 32);
  } else {
    const int shift = i8::row_shift<1>(p);
    uint32_t c[3][4];
    load_chunks<3>(c, p + (k - shift), live ? len - k + shift : 0, len - k < 48);
    i8::merge16(v[0], c[0], c[1], shift);
    i8::merge16(v[1], c[1], c[2], shift);
  }
}
// Place in a ring of stages, and the parity of its "empty" barrier's phase that a writer waits for.
struct Place {
  int s;
  uint32_t ph;
  __device__ __forceinline__ void forward(int steps, int stages) {
    s += steps;
    while (s >= stages) {
      s -= stages;
      ph ^= 1u;
    }
  }
};

}  // namespace mx4

// Pairs of CTAs (kern_mx4_pair.cu), up to kPairGroups groups, whose first tiles and rows lie in their shared memory (256
// groups, 2048 -> 2048: of 256 rows pairs 158 us, tiles 207, of 64 rows 125 and 109); maps: of 128 rows at a time.
constexpr int kPairGroups = 256;
cudaError_t launch_mx4_pair(const Mx4Args& A, const mx4::Maps& maps, cudaStream_t st, int expire);
}  // namespace bk
