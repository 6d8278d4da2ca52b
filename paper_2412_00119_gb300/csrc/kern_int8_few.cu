// kern_int8_few.cu -- the 8-bit product of one to eight rows (a serving step's tokens):
// the weights stream through once.
//
// mma.sync m16n8k32 on 8-bit integers, int32 sums: 16 channels x 8 rows.  Its rate is low on
// sm_103a (75 T products/s), but eight rows need 7.2 us of it beside the 10 us that
// 8192 x 8192 weights take to arrive (dp4a, a third of a warp instruction per clock and SM:
// 13.8 us for one row, 44.6 for eight).  The order of k inside an MMA is free, alike in both
// operands: a lane loads 16 neighbouring codes of a row, four lanes 64, and its words go
// to the places of two MMAs.
// A CTA takes 16 channels, its warps a slice of K each; their sums meet in shared memory.
// The weights come through a ring of the warp's own, 256 codes of the 16 channels at a time
// with asynchronous copies of 256 neighbouring bytes (loads of 64 bytes of 8 rows straight
// into the fragments: 16.3 us for one row); the rows' codes come from L1.
// Bound: the weights' bytes.
#include "int8_common.cuh"
#include "tc_common.cuh"

namespace bk {
namespace {

using namespace i8;

constexpr int kChannels = 16;
constexpr int kStep = 256;        // codes of a row per turn
constexpr int kRing = 3;          // turns of the ring (four: fewer CTAs stay, 18.2 us)

template <int kAlign> struct Few {
  // bytes of a channel per turn: 16 chunks, or 17 (at a pitch of 320, without bank conflicts, fewer
  // CTAs stay: 1 x 8191 -> 8192 28 us)
  static constexpr int kPitch = kAlign == 16 ? 256 : 272;
  static constexpr int kTurnBytes = kChannels * kPitch;
  // place of chunk c of channel r: of odd channels swapped by fours, which puts the 64 bytes of
  // two channels that eight lanes read on different banks
  static __device__ __forceinline__ uint32_t at(int r, int c) {
    return (uint32_t)(r * kPitch + 16 * (kAlign == 16 ? c ^ ((r & 1) << 2) : c));
  }
};

__device__ __forceinline__ void mma_s8(int (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                       uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

template <int kWarps, int kAlign>
__global__ void __launch_bounds__(32 * kWarps) k_int8_few(const Int8Args A) {
  using F = Few<kAlign>;
  extern __shared__ uint4 smem_few[];
  __shared__ int part[kWarps][kChannels * kFewRows];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = lane >> 2, q = lane & 3;    // row of the fragments, 16-byte piece of 64
  const int j0 = (int)blockIdx.x * kChannels;
  const int turns = (A.K + kStep - 1) / kStep;
  const int first = (int)((int64_t)turns * warp / kWarps), last = (int)((int64_t)turns * (warp + 1) / kWarps);
  const uint32_t ring = tc::smem_u32(smem_few) + (uint32_t)(warp * kRing * F::kTurnBytes);
  // copies: half a warp per channel, channels lane / 16, + 2, ..
  const int c0 = lane & 15, r0 = lane >> 4;
  const int8_t* wrow = A.w + (int64_t)(j0 + r0) * A.ldw;
  const int8_t* any = aligned16(A.w);
  // the first turns' weights on their way to L2 while the launch before this one ends (all
  // turns': what is needed first waits behind the rest, 16.0 us in place of 14.0)
  for (int t = first; t < min(last, first + 2); ++t) {
    const int at = kStep * t + 128 * (c0 >> 3);
    if (j0 + r0 + 2 * (c0 & 7) < A.N && at < A.K)
      asm volatile("prefetch.global.L2 [%0];" ::"l"(wrow + (int64_t)(2 * (c0 & 7)) * A.ldw + at));
  }
  pdl_wait();
  pdl_trigger();
  auto copy = [&](int t, uint32_t slot) {
    if (t < last) {
      const uint32_t to = ring + slot * (uint32_t)F::kTurnBytes;
      const int8_t* row = wrow;
#pragma unroll
      for (int i = 0; i < kChannels / 2; ++i, row += 2 * A.ldw)
        copy_chunk(to + F::at(r0 + 2 * i, c0), row, row_shift<kAlign>(row), kStep * t + 16 * c0,
                   j0 + r0 + 2 * i < A.N ? A.K : -16, any);
      if (kAlign != 16 && lane < kChannels) {
        row = A.w + (int64_t)(j0 + lane) * A.ldw;
        copy_chunk(to + F::at(lane, 16), row, row_shift<kAlign>(row), kStep * (t + 1), j0 + lane < A.N ? A.K : -16, any);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int d = 0; d < kRing - 1; ++d) copy(first + d, d);
  // (rows past n read row 0: what comes of them is dropped)
  const int8_t* ar = A.a + (g < A.n ? g : 0) * A.lda;
  const int ashift = row_shift<kAlign>(ar);
  const int shift0 = row_shift<kAlign>(A.w + (int64_t)(j0 + g) * A.ldw);
  const int shift1 = row_shift<kAlign>(A.w + (int64_t)(j0 + g + 8) * A.ldw);
  int acc[2][4] = {};
  uint32_t slot = 0;
#pragma unroll 1
  for (int t = first; t < last; ++t) {
    uint32_t b[4][4];
    if (kStep * (t + 1) + (kAlign == 16 ? 0 : 16) <= A.K) {
#pragma unroll
      for (int h = 0; h < 4; ++h) load16_inside<kAlign>(b[h], ar, ashift, kStep * t + 64 * h + 16 * q);
    } else {
#pragma unroll
      for (int h = 0; h < 4; ++h) load16<kAlign>(b[h], ar, ashift, kStep * t + 64 * h + 16 * q, A.K);
    }
    asm volatile("cp.async.wait_group %0;" ::"n"(kRing - 2) : "memory");
    __syncwarp();   // every lane's copies of this turn, and its reads of the turn before
    copy(t + kRing - 1, slot == 0 ? kRing - 1 : slot - 1);
    const uint32_t from = ring + slot * (uint32_t)F::kTurnBytes;
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      uint32_t x[4], y[4];
      lds_chunk(x, from + F::at(g, 4 * h + q));
      lds_chunk(y, from + F::at(g + 8, 4 * h + q));
      if constexpr (kAlign != 16) {
        uint32_t more[4], v[4];
        lds_chunk(more, from + F::at(g, 4 * h + q + 1));
        merge16(v, x, more, shift0);
        lds_chunk(more, from + F::at(g + 8, 4 * h + q + 1));
        merge16(x, y, more, shift1);
        mma_s8(acc[0], v[0], x[0], v[1], x[1], b[h][0], b[h][1]);
        mma_s8(acc[1], v[2], x[2], v[3], x[3], b[h][2], b[h][3]);
      } else {
        mma_s8(acc[0], x[0], y[0], x[1], y[1], b[h][0], b[h][1]);
        mma_s8(acc[1], x[2], y[2], x[3], y[3], b[h][2], b[h][3]);
      }
    }
    if (++slot == kRing) slot = 0;
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  // [row][channel]
  int* to = part[warp] + (2 * q) * kChannels + g;
  to[0] = acc[0][0] + acc[1][0];
  to[kChannels] = acc[0][1] + acc[1][1];
  to[8] = acc[0][2] + acc[1][2];
  to[kChannels + 8] = acc[0][3] + acc[1][3];
  __syncthreads();
  const int t = (int)threadIdx.x, c = t % kChannels, i = t / kChannels;
  if (t >= kChannels * kFewRows) return;   // (whole warps)
  int s = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) s += part[w][t];
  if (A.words) {
    const bool on = j0 + c < A.N && s >= (A.thr && j0 + c < A.N ? A.thr[j0 + c] : 0);
    const unsigned bits = __ballot_sync(0xffffffffu, on);   // two rows per warp
    if (c == 0 && i < A.n)
      reinterpret_cast<uint16_t*>(A.words + i * ((A.N + 63) / 64))[blockIdx.x] = (uint16_t)(bits >> (t & 16));
  } else if (j0 + c < A.N && i < A.n) {
    put_out(A, i, j0 + c, s);
  }
}

template <int kWarps, int kAlign>
cudaError_t launch_few(const Int8Args& A, int ctas, cudaStream_t st) {
  constexpr int kSmem = kWarps * kRing * Few<kAlign>::kTurnBytes;
  static std::atomic<uint64_t> done{0};
  const cudaError_t e = allow_smem(done, k_int8_few<kWarps, kAlign>, kSmem);
  if (e != cudaSuccess) return e;
  return launch_kernel(k_int8_few<kWarps, kAlign>, dim3((unsigned)ctas), dim3(32 * kWarps), (size_t)kSmem, st, true, A);
}

template <int kAlign>
cudaError_t launch_slices(const Int8Args& A, cudaStream_t st) {
  // signs: every part of the words, also past N
  const int ctas = A.words ? 4 * (A.N / 64 + (A.N % 64 != 0)) : A.N / kChannels + (A.N % kChannels != 0);
  // slices of K: a dozen warps an SM, a turn at least for each
  const int turns = (A.K + kStep - 1) / kStep, want = 12 * sm_count();
  if (turns < 8 || (int64_t)4 * ctas >= want) return launch_few<4, kAlign>(A, ctas, st);
  if (turns < 16 || (int64_t)8 * ctas >= want || kAlign != 16) return launch_few<8, kAlign>(A, ctas, st);
  return launch_few<kAlign == 16 ? 16 : 8, kAlign>(A, ctas, st);
}

}  // namespace

cudaError_t launch_int8_few(const Int8Args& A, cudaStream_t st) {
  return operand_align(A) == 16 ? launch_slices<16>(A, st) : launch_slices<1>(A, st);
}

}  // namespace bk
