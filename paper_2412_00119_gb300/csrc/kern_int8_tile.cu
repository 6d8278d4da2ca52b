// kern_int8_tile.cu -- the 8-bit product on the tensor cores, tiles of one CTA.
//
// tcgen05 has no 8-bit integer kind on sm_103a.  A code is exact in fp16, the product
// of two is an integer of at most 2^14, and fp32 holds every partial sum of 1024 of
// them exactly (2^24), so kind::f16 gives S exactly if the accumulators are taken
// to int32 every 1024 k at most.  They are double-buffered in tensor memory: one
// chunk's sums are added to int32 registers while the next chunk's MMAs run.
//
// A CTA computes 128 channels (MMA M; lanes of tensor memory) x NT rows (MMA N) over
// its share of K; the CTAs of a cluster share K, and send each other int32 sums through
// distributed shared memory (integers: any order gives the same).  Channels on M: a
// narrow batch costs narrow MMAs, and a warp's lanes hold 32 neighbouring channels of a row,
// as the output wants them; for many rows and few channels the two change places
// (17,871 x 4646 -> 78 158 us, swapped 32).  Warps of a CTA:
//   - 16 workers in four groups that take the k-steps (128 codes of every row, or 64) in
//     turn: a warp copies its rows' codes kDeep turns ahead (asynchronous copies to a ring
//     of its own: with loads to registers, whose scoreboards are few, 26 us for 32 rows of
//     8192 -> 8192, now 16.7), turns them into fp16, the weights into tensor memory (a lane per
//     channel) and the activations into shared memory (128B swizzle), and arrives on "full";
//     between them the workers drain finished chunks;
//   - one or two warps issue the MMAs (two: of even and odd k-steps, each into accumulators
//     of its own), committing to "empty" per k-step and "done" per chunk;
//   - with activations that are ready as fp16 blocks (more than 32 rows) one thread copies
//     those, the workers start on the weights while the launch that writes the blocks runs,
//     and 100 x 4096 -> 8192 takes 15.4 us (19.0 with the workers making them).
// Bound, up to 32 rows: the workers' instructions, then the weights' bytes (a k-step of 128
// 620 clocks, 8192 x 8192 weights 4.1 TB/s).  At 128 ready rows: shared memory's 128 bytes per
// clock (96 KB per k-step of 128, 790 clocks where its MMAs need 512).  (With the fp16
// weights in shared memory too a k-step of 64 took 570 clocks at 32 rows and 750 at 128.)  What
// follows the last sum, the exchange between CTAs above all, takes 2 to 3 us of every call.
// Every wait is bounded; if one expires the CTA's partial sums are made again on CUDA
// cores, so the output is always whole.
#include <algorithm>
#include <type_traits>
#include <utility>

#include "int8_common.cuh"
#include "tc_common.cuh"

namespace bk {
namespace {

using namespace tc;
using namespace i8;

constexpr int CM = 128;                 // channels of a tile
constexpr int kWorkers = 16;
constexpr int kFewTiles = 12;           // tiles at most whose K eight CTAs share (more clusters of eight find no room at once)
constexpr int kGroups = 4;              // worker groups, each a k-step of its own
constexpr int kSmemBytes = 225 * 1024;  // for stages and copies in flight

template <int NT, int kAlign, bool kReady> struct Cfg {
  static constexpr int kSub = NT <= 64 || kReady ? 2 : 1;      // 64 codes (a 128-byte row of fp16) each
  static constexpr int kStep = 64 * kSub;                      // codes of a k-step
  static constexpr int kIssuers = NT <= 64 ? 2 : 1;
  static constexpr int kThreads = 32 * (kWorkers + kIssuers + (kReady ? 1 : 0));
  static constexpr int kChunk = 1024 / kStep * kIssuers;       // k-steps between drains: 1024 k per accumulator
  // a row of the ring: chunks of 16 codes, one more where they are merged (int8_common.cuh)
  static constexpr int kRow = kStep + (kAlign == 16 ? 0 : 16);
  static constexpr int kTurnRows = 32 + (kReady ? 0 : NT / 4); // rows of a warp: channels, activations
  static constexpr int kTurnBytes = kWorkers * kTurnRows * kRow;
  static constexpr int kStageBytes = NT * 128 * kSub;          // activations
  static constexpr int kStageCols = 32 * kSub;                 // weights
  static constexpr int kAccCols = 2 * kIssuers * NT;
  static constexpr int stages(int deep) {
    return std::min((512 - kAccCols) / kStageCols, std::min(8, (kSmemBytes - deep * kTurnBytes) / kStageBytes)) / 2 * 2;
  }
  // Turns in flight, and stages: at least one per group, and a stage always the same
  // issuer's.  (A warp that waits for its stage's last use has seen the k-step kGroups +
  // kStages back consumed; with fewer stages that says nothing of the use before the last,
  // whose phase has the same parity.)
  static constexpr int kDeep = stages(4) >= kGroups ? 4 : (stages(3) >= kGroups ? 3 : (stages(2) >= kGroups ? 2 : 1));
  static constexpr int kRingBytes = kDeep * kTurnBytes;
  static constexpr int kStages = stages(kDeep);
  static constexpr int kTmemCols = kAccCols + kStageCols * kStages <= 256 ? 256 : 512;
  static constexpr int kCols = NT / 4;                         // accumulator columns (rows) of a worker
  static_assert(kAccCols + kStageCols * kStages <= 512, "tensor memory");
  static_assert(4 * CM * NT <= kStages * kStageBytes + kRingBytes, "exchange fits");
  static_assert(kStages >= kGroups && kStages <= kChunk, "a chunk is drained before the one after the next starts");
  // Place of chunk c of row r of the ring, from its row's start: swapped so that eight lanes
  // that read a chunk of eight rows are on different banks (rows of 80 and 144 bytes are by
  // themselves).
  static __device__ __forceinline__ int chunk_at(int r, int c) {
    return 16 * (kAlign != 16 ? c : (kSub == 2 ? c ^ (r & 7) : c ^ ((r >> 1) & 3)));
  }
};

struct __align__(8) TileShared {
  unsigned long long full[8], empty[8];
  unsigned long long done[2], drained[2];
  unsigned long long left, never;
  uint32_t tmem_base;
  int failed, left_failed;
};

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// What a thread's outputs need from memory: asked for before the sums are there.
struct Factors {
  float sw, bias, sa;
  int thr;
};

// Outputs of a worker warp where the lanes are rows and a thread has kRows channels from i on
// of its own (swapped operands); end: the tile's last channel + 1.  patch: shared memory of the
// warp's (kPatch bytes), through which rows at odd places are written with the lanes along them
// (10,868 x 832 -> 521 bf16 28 us; by single values of the lane's own row 66).
constexpr int kPatch = 32 * 33 * 4;
template <int kRows>
__device__ __forceinline__ void write_channels(const Int8Args& A, const int (&v)[kRows], int64_t i, int64_t end, int jw,
                                               const Factors& F, uint32_t* patch) {
  static_assert(kRows >= 8 && 32 % kRows == 0, "whole bytes of signs");
  const int lane = (int)(threadIdx.x & 31), j = jw + lane;
  const int live = (int)max((int64_t)0, min((int64_t)kRows, A.n - i));   // channels that are some
  if (A.words) {
    const int64_t nw = (A.n + 63) / 64;
    uint32_t bits = 0u;
#pragma unroll
    for (int e = 0; e < kRows; ++e) bits |= v[e] >= __shfl_sync(kFull, F.thr, e) ? 1u << e : 0u;
    bits &= live >= 32 ? 0xFFFFFFFFu : (1u << live) - 1u;
    if (j < A.N && i < 64 * nw) {
      uint8_t* to = reinterpret_cast<uint8_t*>(A.words + j * nw) + (i >> 3);
      if constexpr (kRows == 32) *reinterpret_cast<uint32_t*>(to) = bits;
      else if constexpr (kRows == 16) *reinterpret_cast<uint16_t*>(to) = (uint16_t)bits;
      else *to = (uint8_t)bits;
      // (tiles of 32 may end in the middle of a row's last word: the rest is zero)
      if (i + kRows == end && end >= A.n && end < 64 * nw) *reinterpret_cast<uint32_t*>(to + kRows / 8) = 0u;
    }
    return;
  }
  auto store = [&](auto* out) {
    using T = std::remove_pointer_t<decltype(out)>;
    constexpr int kVec = 16 / (int)sizeof(T);
    T y[kRows];
    const bool has_bias = A.bias != nullptr;
#pragma unroll
    for (int e = 0; e < kRows; ++e) {
      if constexpr (std::is_same<T, int32_t>::value) {
        y[e] = v[e];
      } else {
        const float f = scaled((float)v[e], F.sw, __shfl_sync(kFull, F.sa, e)), b = __shfl_sync(kFull, F.bias, e);
        y[e] = out_cast<T>(has_bias ? __fadd_rn(f, b) : f);
      }
    }
    T* first = out + (int64_t)jw * A.ldo + i;
    if (live == kRows && ((reinterpret_cast<uintptr_t>(first) | (uintptr_t)(A.ldo * (int64_t)sizeof(T))) & 15) == 0) {
      T* p = first + (int64_t)lane * A.ldo;
#pragma unroll
      for (int e = 0; e < kRows; e += kVec) {
        union { uint4 w; T e[kVec]; } u;
#pragma unroll
        for (int x = 0; x < kVec; ++x) u.e[x] = y[e + x];
        if (j < A.N) *reinterpret_cast<uint4*>(p + e) = u.w;
      }
    } else {
#pragma unroll
      for (int e = 0; e < kRows; ++e) *reinterpret_cast<T*>(patch + lane * (kRows + 1) + e) = y[e];
      __syncwarp();
      constexpr int kAcross = 32 / kRows;   // rows of an instruction
      const int e = lane % kRows;
#pragma unroll 8
      for (int r = lane / kRows; r < 32; r += kAcross)
        if (jw + r < A.N && e < live) first[(int64_t)r * A.ldo + e] = *reinterpret_cast<const T*>(patch + r * (kRows + 1) + e);
    }
  };
  switch (A.type) {
    case BMLP_F32: store(static_cast<float*>(A.out)); break;
    case BMLP_F16: store(static_cast<__half*>(A.out)); break;
    case BMLP_BF16: store(static_cast<__nv_bfloat16*>(A.out)); break;
    default: store(static_cast<int32_t*>(A.out));
  }
}

// Outputs of a worker warp from its registers: kRows rows from i on of 32 channels from jw on,
// a lane per channel.
template <int kRows>
__device__ __forceinline__ void write_rows(const Int8Args& A, const int (&v)[kRows], int64_t i, int jw, const Factors& F) {
  const int lane = threadIdx.x & 31, j = jw + lane;
  const int rows = (int)max((int64_t)0, min((int64_t)kRows, A.n - i));
  if (A.words) {
    const int nw32 = 2 * ((A.N + 63) / 64);
    uint32_t mine = 0u;
#pragma unroll
    for (int e = 0; e < kRows; ++e) {
      const uint32_t w = __ballot_sync(kFull, j < A.N && v[e] >= F.thr);
      if (lane == e) mine = w;
    }
    if (lane < rows && (jw >> 5) < nw32) reinterpret_cast<uint32_t*>(A.words)[(i + lane) * nw32 + (jw >> 5)] = mine;
    return;
  }
  auto store = [&](auto* out) {
    using T = std::remove_pointer_t<decltype(out)>;
    T* p = out + i * A.ldo + j;
    const bool has_bias = A.bias != nullptr;
#pragma unroll
    for (int e = 0; e < kRows; ++e, p += A.ldo) {
      const float sa = __shfl_sync(kFull, F.sa, e);
      T y;
      if constexpr (std::is_same<T, int32_t>::value) {
        y = v[e];
      } else {
        const float f = scaled((float)v[e], sa, F.sw);
        y = out_cast<T>(has_bias ? __fadd_rn(f, F.bias) : f);
      }
      if (e < rows && j < A.N) *p = y;
    }
  };
  switch (A.type) {
    case BMLP_F32: store(static_cast<float*>(A.out)); break;
    case BMLP_F16: store(static_cast<__half*>(A.out)); break;
    case BMLP_BF16: store(static_cast<__nv_bfloat16*>(A.out)); break;
    default: store(static_cast<int32_t*>(A.out));
  }
}

// The S CTAs of a cluster each finish kCols / S of every worker's columns: a thread sends the
// partial sums of the others' columns to the same thread there (stores: nothing waits for
// them), and adds what it was sent.  Slot of a sender: its distance from the receiver.
template <int kCols, int S>
__device__ __forceinline__ void exchange_and_write(const Int8Args& A, const int (&acc)[kCols], uint8_t* smem, uint32_t rank,
                                                   int64_t i0, int jw, const Factors& F) {
  constexpr int kOwn = kCols / S, kWide = kOwn % 4 == 0 ? 4 : (kOwn % 2 == 0 ? 2 : 1);
  static_assert(kOwn * S == kCols, "columns are shared out evenly");
  const int tid = (int)threadIdx.x, warp = tid >> 5;
  int own[kOwn];
  const bool worker = warp < kWorkers;
  if constexpr (S == 1) {
#pragma unroll
    for (int e = 0; e < kOwn; ++e) own[e] = acc[e];
  } else {
    cluster_wait();   // every CTA of the cluster is done with its stages and ring
    // kWide columns of a thread side by side, a row of threads, the next kWide
    const uint32_t base = smem_u32(smem) + (uint32_t)(4 * kWide * tid);
    if (worker) {
#pragma unroll
      for (int q = 0; q < S; ++q) {
        if ((uint32_t)q != rank) {
          const uint32_t slot = ((rank - (uint32_t)q) & (S - 1)) - 1u;
          uint32_t to;
          asm volatile("mapa.shared::cluster.u32 %0, %1, %2;"
                       : "=r"(to) : "r"(base + slot * (uint32_t)(kOwn * 4 * 32 * kWorkers)), "r"(q));
#pragma unroll
          for (int e = 0; e < kOwn; e += kWide) {
            const uint32_t at = to + (uint32_t)(e * 4 * 32 * kWorkers);
            const int* v = acc + q * kOwn + e;
            if constexpr (kWide == 4)
              asm volatile("st.shared::cluster.v4.s32 [%0], {%1, %2, %3, %4};"
                           ::"r"(at), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
            else if constexpr (kWide == 2)
              asm volatile("st.shared::cluster.v2.s32 [%0], {%1, %2};" ::"r"(at), "r"(v[0]), "r"(v[1]) : "memory");
            else
              asm volatile("st.shared::cluster.s32 [%0], %1;" ::"r"(at), "r"(v[0]) : "memory");
          }
        }
      }
#pragma unroll
      for (int q = 0; q < S; ++q)
        if ((uint32_t)q == rank) {
#pragma unroll
          for (int e = 0; e < kOwn; ++e) own[e] = acc[q * kOwn + e];
        }
    }
    cluster_arrive();
    cluster_wait();   // what was sent is there; nobody writes to another CTA after this
    if (worker) {
#pragma unroll
      for (int x = 0; x < S - 1; ++x)
#pragma unroll
        for (int e = 0; e < kOwn; ++e)
          own[e] += reinterpret_cast<const int*>(smem)[(x * kOwn + e / kWide * kWide) * 32 * kWorkers + kWide * tid + e % kWide];
    }
  }
  if (worker) {
    const int64_t i = i0 + kCols * (warp >> 2) + kOwn * (int)rank;
    if constexpr (kOwn >= 8) {
      if (A.swapped) {
        // (past what the cluster's other CTAs write)
        uint32_t* patch = reinterpret_cast<uint32_t*>(smem + (S - 1) * kOwn * 128 * kWorkers + warp * kPatch);
        write_channels<kOwn>(A, own, i, i0 + 4 * kCols, jw, F, patch);
        return;
      }
    }
    write_rows<kOwn>(A, own, i, jw, F);
  }
}

// kReady: the activations as fp16 blocks (kern_int8_pair.cu), written by the launch before
// this one, which writes nothing else that is read here.
template <int NT, int kAlign, bool kReady>
__global__ void __launch_bounds__(Cfg<NT, kAlign, kReady>::kThreads, 1)
    k_int8_tile(const Int8Args A, const uint8_t* __restrict__ ablocks, int split, int expire) {
  using C = Cfg<NT, kAlign, kReady>;
  constexpr int kStages = C::kStages, kDeep = C::kDeep, kIssuers = C::kIssuers, kChunk = C::kChunk;
  // a warp's copies: units of kUnit rows, 4 kSub lanes per row
  constexpr int kSub = C::kSub, kUnit = 8 / kSub;
  constexpr int kUnitsA = 32 / kUnit, kUnitsB = kReady ? 0 : NT / 4 / kUnit, kUnits = kUnitsA + kUnitsB;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  uint8_t* ring = base + kStages * C::kStageBytes;
  TileShared* sh = reinterpret_cast<TileShared*>(ring + C::kRingBytes);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = split > 1 ? cluster_rank() : 0u;
  const int j0 = (int)(blockIdx.x / (unsigned)split) * CM;
  const int64_t i0 = (int64_t)blockIdx.y * NT;
  volatile int* failed = &sh->failed;
  // this CTA's k-steps
  const int all = (A.K + C::kStep - 1) / C::kStep;
  const int first = (int)((int64_t)all * rank / split), steps = (int)((int64_t)all * (rank + 1) / split) - first;
  const int chunks = (steps + kChunk - 1) / kChunk;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&sh->full[s], kWorkers / kGroups + (kReady ? 1 : 0));
      mbar_init(&sh->empty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&sh->done[b], kIssuers);
      mbar_init(&sh->drained[b], kWorkers);
    }
    mbar_init(&sh->left, kIssuers);
    mbar_init(&sh->never, 1);
    sh->failed = sh->left_failed = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kWorkers) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                 ::"r"(smem_u32(&sh->tmem_base)), "r"(C::kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = sh->tmem_base;
  // A warp's rows of a k-step: channels 32 q .. + 31 of the tile and NT / 4 activation rows.
  const int grp = warp >> 2, q = warp & 3;
  const int r = lane / (4 * kSub), c = lane % (4 * kSub);   // copies: row of a unit, 16 of its codes
  const int ja = j0 + 32 * q + r;                 // channel, + kUnit per unit
  const int64_t ib = i0 + NT / 4 * q + r;         // row, + kUnit per unit
  if constexpr (!kReady) {
    if (warp < kWorkers && c == 0) {
      // the first turn's weights on their way to L2 while the launch before this one ends
      const int k = C::kStep * (first + grp);
#pragma unroll
      for (int u = 0; u < kUnitsA; ++u)
        if (ja + kUnit * u < A.N && k < A.K)
          asm volatile("prefetch.global.L2 [%0];" ::"l"(A.w + (int64_t)(ja + kUnit * u) * A.ldw + k));
    }
    pdl_wait();
    pdl_trigger();
  } else if (warp >= kWorkers) {
    pdl_wait();   // (the workers' copies of the weights need not wait)
  }

  Factors F = {};
  constexpr int kCols = C::kCols;
  int acc[kCols];
#pragma unroll
  for (int e = 0; e < kCols; ++e) acc[e] = 0;
  if (warp < kWorkers) {
    // ---------------- workers ----------------
    const int8_t* wrow = A.w + (int64_t)ja * A.ldw;
    const int8_t* arow = A.a + ib * A.lda;
    const int8_t* any = aligned16(A.w);
    const int64_t wstep = kUnit * A.ldw, astep = kUnit * A.lda;
    uint8_t* const mine = ring + warp * kDeep * C::kTurnRows * C::kRow;
    const uint32_t ring_to = smem_u32(mine) + (uint32_t)(r * C::kRow);
    auto copy = [&](int ks, int slot) {
      if (ks < steps) {
        const int k = C::kStep * (first + ks) + 16 * c;
        const uint32_t to = ring_to + (uint32_t)(slot * C::kTurnRows * C::kRow);
        // (a unit of four rows: the swap by the row's low bits alternates between two places)
        if (C::kStep * (first + ks + 1) + (kAlign == 16 ? 0 : 16) <= A.K) {
          // every code inside its row; channels past N and rows past n as zeros, with nothing read
          // (18 rows of 4863 -> 12288 28 us; 45 where the 14 others read the tile's first row, a line
          // that every CTA then asks for many times a k-step)
          const int8_t* row = wrow + k;
#pragma unroll
          for (int u = 0; u < kUnits; ++u) {
            if (u == kUnitsA) row = arow + k;
            const bool live = u < kUnitsA ? ja + kUnit * u < A.N : ib + kUnit * (u - kUnitsA) < A.n;
            const int8_t* p = live ? row : any;
            const int size = live ? 16 : 0;
            if constexpr (kAlign != 16) p = aligned16(p);
            const uint32_t unit = to + (uint32_t)(u * kUnit * C::kRow);
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;"
                         ::"r"(unit + (uint32_t)C::chunk_at(kUnit == 4 ? r + 4 * (u & 1) : r, c)), "l"(p), "r"(size) : "memory");
            if (kAlign != 16 && c == 0)
              asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;"
                           ::"r"(unit + (uint32_t)C::kStep), "l"(p + (live ? C::kStep : 0)), "r"(size) : "memory");
            row += u < kUnitsA ? wstep : astep;
          }
        } else {
          const int8_t* row = wrow;
#pragma unroll
          for (int u = 0; u < kUnits; ++u) {
            if (u == kUnitsA) row = arow;
            const bool live = u < kUnitsA ? ja + kUnit * u < A.N : ib + kUnit * (u - kUnitsA) < A.n;
            const int shift = row_shift<kAlign>(row);
            const uint32_t unit = to + (uint32_t)(u * kUnit * C::kRow);
            copy_chunk(unit + (uint32_t)C::chunk_at(kUnit == 4 ? r + 4 * (u & 1) : r, c), row, shift, k, live ? A.K : -16, any);
            if (kAlign != 16 && c == 0)
              copy_chunk(unit + (uint32_t)C::kStep, row, shift, k + C::kStep, live ? A.K : -16, any);
            row += u < kUnitsA ? wstep : astep;
          }
        }
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int d = 0; d < kDeep; ++d) copy(grp + kGroups * d, d);
    // reads: a lane per channel; of the activations a row rb of a unit and a chunk cb, eight
    // lanes (which meet in shared memory) two rows and, of 128 codes, a half of each
    const uint8_t* const read_w = mine + lane * C::kRow;
    const int rb = kSub == 2 ? 2 * (lane >> 4) + ((lane >> 2) & 1) : r;
    const int cb = kSub == 2 ? 4 * (((lane >> 3) ^ (lane >> 2)) & 1) + (lane & 3) : c;
    const uint8_t* const read_a = mine + (32 + rb) * C::kRow;
    const int wshift = row_shift<kAlign>(A.w + (int64_t)(j0 + 32 * q + lane) * A.ldw);
    // 32 bytes of fp16 per piece: chunks 2 (cb % 4) and one more of the row, swizzled (the swizzle
    // goes by the row's low three bits: a unit of four alternates, as above)
    uint8_t* const at = base + (cb >> 2) * (NT * 128) + 128 * (NT / 4 * q + rb);
    const int swz0 = (32 * (cb & 3)) ^ (16 * (rb & 7));
    const uint32_t lanes = (uint32_t)(32 * q) << 16;
    const uint32_t tacc = tmem + ((uint32_t)(32 * (warp & 3)) << 16) + (uint32_t)(kCols * (warp >> 2));
    int drained = 0;   // chunks added to acc
    bool arrived = false;
    bool ok = true;
    auto drain = [&]() {
      const int b = drained & 1;
      ok = __all_sync(kFull, mbar_wait(&sh->done[b], (uint32_t)(drained >> 1) & 1u, failed));
      if (!ok) return;
      if (split > 1 && drained == chunks - 1) {
        // with the last MMAs stages and ring are done with: the others may write there
        cluster_arrive();
        arrived = true;
      }
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      // (the odd k-steps' accumulator has nothing in a chunk of one)
      const int both = min(kIssuers, steps - drained * kChunk);
#pragma unroll 1
      for (int m = 0; m < both; ++m)
#pragma unroll
        for (int e = 0; e < kCols; e += kCols % 16 == 0 ? 16 : 8) {
          if constexpr (kCols % 16 == 0) {
            uint32_t v[16];
            tmem_load16(v, tacc + (uint32_t)((kIssuers * b + m) * NT + e));
            tmem_wait_ld(v);
#pragma unroll
            for (int x = 0; x < 16; ++x) acc[e + x] += __float2int_rn(__uint_as_float(v[x]));
          } else {
            uint32_t v[8];
            tmem_load8(v, tacc + (uint32_t)((kIssuers * b + m) * NT + e));
#pragma unroll
            for (int x = 0; x < 8; ++x) acc[e + x] += __float2int_rn(__uint_as_float(v[x]));
          }
        }
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh->drained[b]);
      ++drained;
    };
    uint32_t s = (uint32_t)grp, ph = 1;
    auto wrap = [&]() {
      while (s >= (uint32_t)kStages) {
        s -= kStages;
        ph ^= 1u;
      }
    };
    wrap();
    int slot = 0;
#pragma unroll 1
    for (int ks = grp; ks < steps && ok; ks += kGroups) {
      if (ks >= (drained + 1) * kChunk + kStages) {
        drain();
        if (!ok) break;
      }
      ok = __all_sync(kFull, mbar_wait(&sh->empty[s], ph, failed));
      if (!ok) break;
      asm volatile("cp.async.wait_group %0;" ::"n"(kDeep - 1) : "memory");
      __syncwarp();   // (pieces that other lanes copied)
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      const int turn = slot * C::kTurnRows * C::kRow;
      const uint32_t tw = tmem + lanes + (uint32_t)C::kAccCols + (uint32_t)C::kStageCols * s;
      {
        // the row's words: whole chunks, or from the 8 bytes on that hold the first code, a word or
        // none of which is passed over, and then shifted by bytes (merge16's steps, the first by
        // address: 17,871 x 4646 -> 78 30 us, by merge16 32)
        constexpr int kWords = 16 * kSub + (kAlign == 16 ? 0 : 2);
        uint32_t v[kWords];
        if constexpr (kAlign == 16) {
#pragma unroll
          for (int i = 0; i < kWords / 4; ++i) {
            const uint4 w = *reinterpret_cast<const uint4*>(read_w + turn + C::chunk_at(lane, i));
            v[4 * i] = w.x, v[4 * i + 1] = w.y, v[4 * i + 2] = w.z, v[4 * i + 3] = w.w;
          }
        } else {
          const uint8_t* from = read_w + turn + (wshift & 8);
#pragma unroll
          for (int i = 0; i < kWords / 2; ++i) {
            const uint2 w = *reinterpret_cast<const uint2*>(from + 8 * i);
            v[2 * i] = w.x, v[2 * i + 1] = w.y;
          }
#pragma unroll
          for (int i = 0; i < kWords - 1; ++i) v[i] = wshift & 4 ? v[i + 1] : v[i];
#pragma unroll
          for (int i = 0; i < kWords - 2; ++i) v[i] = __funnelshift_r(v[i], v[i + 1], 8u * (uint32_t)(wshift & 3));
        }
#pragma unroll
        for (int h = 0; h < 2 * kSub; ++h) {
          uint32_t f[16];
#pragma unroll
          for (int e = 0; e < 8; ++e) codes_f16(v[8 * h + e], f[2 * e], f[2 * e + 1]);
          tmem_store16(tw + 16u * h, f);
        }
      }
      uint8_t* const to = at + s * (uint32_t)C::kStageBytes;
#pragma unroll
      for (int u = 0; u < kUnitsB; ++u) {
        const int high = kUnit == 4 ? 4 * (u & 1) : 0;   // of the row's low three bits
        const uint8_t* from = read_a + turn + u * kUnit * C::kRow;
        const uint4 lo = *reinterpret_cast<const uint4*>(from + C::chunk_at(rb + high, cb));
        uint32_t x[4] = {lo.x, lo.y, lo.z, lo.w};
        if constexpr (kAlign != 16) {
          const uint4 hi = *reinterpret_cast<const uint4*>(from + 16 * cb + 16);
          const uint32_t l[4] = {lo.x, lo.y, lo.z, lo.w}, m[4] = {hi.x, hi.y, hi.z, hi.w};
          merge16(x, l, m, row_shift<kAlign>(A.a + (i0 + NT / 4 * q + rb + kUnit * u) * A.lda));
        }
        uint8_t* const row = to + 128 * kUnit * u;
        uint4 h;
        codes_f16(x[0], h.x, h.y);
        codes_f16(x[1], h.z, h.w);
        *reinterpret_cast<uint4*>(row + (swz0 ^ (16 * high))) = h;
        codes_f16(x[2], h.x, h.y);
        codes_f16(x[3], h.z, h.w);
        *reinterpret_cast<uint4*>(row + (swz0 ^ (16 * high) ^ 16)) = h;
      }
      asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh->full[s]);
      copy(ks + kGroups * kDeep, slot);
      if (++slot == kDeep) slot = 0;
      s += kGroups;
      wrap();
    }
    asm volatile("cp.async.wait_all;" ::: "memory");   // no copy outlives its thread
    if constexpr (kReady) {
      pdl_wait();
      pdl_trigger();
    }
    // what the outputs need, while the last MMAs run
    const int j = j0 + 32 * q + lane;
    F.sw = j < A.N && A.w_scale ? A.w_scale[j] : 1.0f;
    // (lane e: the warp's row e)
    const int own = kCols / split;
    const int64_t i = i0 + kCols * (warp >> 2) + own * (int)rank + lane;
    const bool row = lane < own && i < A.n;
    F.sa = A.a_scale && row ? A.a_scale[i] : 1.0f;
    // (bias and thresholds go with the call's channels)
    const int64_t channel = A.swapped ? i : (int64_t)j;
    const bool some = A.swapped ? row : j < A.N;
    F.bias = some && A.bias ? A.bias[channel] : 0.0f;
    F.thr = some && A.thr ? A.thr[channel] : 0;
    while (ok && drained < chunks) drain();
    if (split > 1 && !arrived) cluster_arrive();   // (after a failure: no copy of this warp is in flight)
    if (expire && threadIdx.x == 0) *failed = 1;
  } else if (kReady && warp == kWorkers + kIssuers) {
    // ---------------- copies of the activations' blocks ----------------
    if (lane == 0) {
      const int nkb = (A.K + 63) / 64;
      const uint8_t* src = ablocks + i0 / 128 * nkb * (int64_t)16384 + i0 % 128 * 128;
      uint32_t s = 0, ph = 1;
      bool ok = true;
#pragma unroll 1
      for (int ks = 0; ks < steps; ++ks) {
        ok = mbar_wait(&sh->empty[s], ph, failed);
        if (!ok) break;
        const int kb = kSub * (first + ks), subs = min(kSub, nkb - kb);   // (a last k-step's second 64: none)
        mbar_arrive_tx(&sh->full[s], (uint32_t)(subs * NT * 128));
        for (int x = 0; x < subs; ++x)
          bulk_g2s(base + s * C::kStageBytes + x * (NT * 128), src + (int64_t)(kb + x) * 16384, NT * 128, &sh->full[s]);
        if (++s == (uint32_t)kStages) {
          s = 0;
          ph ^= 1u;
        }
      }
      if (!ok) {
        // no copy outlives the CTA: what was asked for lands long before this wait's limit
        mbar_wait(&sh->never, 0, &sh->left_failed, 2000000ull);
      }
    }
  } else {
    // ---------------- MMA issuers ----------------
    const int m = warp - kWorkers;
    const bool lead = elect_one();
    const uint32_t t0 = uniform(tmem), d = t0 + (uint32_t)(m * NT);
    const uint64_t desc0 = smem_desc(uniform(smem_u32(base)));
    constexpr uint32_t kIdesc = idesc_f16(CM, NT);
    uint32_t s = (uint32_t)m, ph = 0;
    bool ok = true;
#pragma unroll 1
    for (int ch = 0; ch < chunks && ok; ++ch) {
      const int b = ch & 1;
      if (ch >= 2) {
        ok = __all_sync(kFull, mbar_wait(&sh->drained[b], (uint32_t)((ch >> 1) - 1) & 1u, failed));
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      }
      const int end = min(steps, (ch + 1) * kChunk);
      uint32_t accumulate = 0u;
#pragma unroll 1
      for (int ks = ch * kChunk + m; ks < end && ok; ks += kIssuers) {
        ok = __all_sync(kFull, mbar_wait(&sh->full[s], ph, failed));
        if (!ok) break;
        // the workers' stores to shared memory, acquired above, before the MMAs' reads
        if constexpr (!kReady) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint64_t bd = desc0 + (uint64_t)(s * (uint32_t)(C::kStageBytes >> 4));
        const uint32_t ta = t0 + (uint32_t)C::kAccCols + (uint32_t)C::kStageCols * s;
        // (ready activations of a last k-step may end after its first 64)
        const int mmas = kReady && kSub * (first + ks) + 1 >= (A.K + 63) / 64 ? 4 : 4 * kSub;
        if (lead) {
#pragma unroll
          for (int e = 0; e < 4 * kSub; ++e)
            if (e < 4 || e < mmas)
              mma_f16_ts(d + (uint32_t)(kIssuers * b * NT), ta + 8 * e, bd + (uint64_t)((e >> 2) * (NT * 128 >> 4) + 2 * (e & 3)),
                         kIdesc, e > 0 ? 1u : accumulate);
          mma_commit(&sh->empty[s]);
        }
        accumulate = 1u;
        s += kIssuers;
        if (s >= (uint32_t)kStages) {
          s -= kStages;
          ph ^= 1u;
        }
      }
      if (ok && lead) mma_commit(&sh->done[b]);
      __syncwarp();
    }
    if (lead) {
      // no MMA outlives its operands and its tensor memory
      mma_commit(&sh->left);
      mbar_wait(&sh->left, 0, &sh->left_failed);
    }
    __syncwarp();
  }
  __syncwarp();
  if (split > 1 && warp >= kWorkers) cluster_arrive();
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  if (warp == kWorkers)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(C::kTmemCols) : "memory");
  if (*failed && warp < kWorkers) {
    // partial sums of this CTA's k range on CUDA cores
    const int k0 = C::kStep * first, k1 = min(A.K, C::kStep * (first + steps)), j = j0 + 32 * q + lane;
#pragma unroll
    for (int e = 0; e < kCols; ++e) {
      const int64_t i = i0 + kCols * (warp >> 2) + e;
      acc[e] = j < A.N && i < A.n ? plain_sum(A.a + i * A.lda, A.w + (int64_t)j * A.ldw, k0, k1) : 0;
    }
  }
  const int jw = j0 + 32 * q;
  switch (split) {
    case 1: exchange_and_write<kCols, 1>(A, acc, base, rank, i0, jw, F); break;
    case 2: exchange_and_write<kCols, 2>(A, acc, base, rank, i0, jw, F); break;
    case 8: exchange_and_write<kCols, 8>(A, acc, base, rank, i0, jw, F); break;
    default: exchange_and_write<kCols, 4>(A, acc, base, rank, i0, jw, F);
  }
}

template <int NT, int kAlign, bool kReady>
cudaError_t launch_tile(const Int8Args& A, const uint8_t* ablocks, int split, int expire, cudaStream_t st) {
  using C = Cfg<NT, kAlign, kReady>;
  constexpr int kSmem = 1024 + C::kStages * C::kStageBytes + C::kRingBytes + (int)sizeof(TileShared);
  static std::atomic<uint64_t> done{0};
  const cudaError_t e = allow_smem(done, k_int8_tile<NT, kAlign, kReady>, kSmem);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((A.N + CM - 1) / CM * split), (unsigned)((A.n + NT - 1) / NT));
  cfg.blockDim = dim3(C::kThreads);
  cfg.dynamicSmemBytes = kSmem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim = {(unsigned)split, 1u, 1u};
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, k_int8_tile<NT, kAlign, kReady>, A, ablocks, split, expire);
}

template <int kAlign>
cudaError_t launch_rows(const Int8Args& A, const uint8_t* ablocks, int nt, int split, int expire, cudaStream_t st) {
  if (ablocks)
    return nt == 64 ? launch_tile<64, kAlign, true>(A, ablocks, split, expire, st)
                    : launch_tile<128, kAlign, true>(A, ablocks, split, expire, st);
  return nt == 32   ? launch_tile<32, kAlign, false>(A, nullptr, split, expire, st)
         : nt == 64 ? launch_tile<64, kAlign, false>(A, nullptr, split, expire, st)
                    : launch_tile<128, kAlign, false>(A, nullptr, split, expire, st);
}

}  // namespace

// Up to four: as many as leave every SM at most one, with eight k-steps of 64 each; of swapped
// operands a thread keeps eight channels (a byte of signs).  Eight for a few tiles (us: 20 rows of
// 8192 -> 512 6.5, by four 9.2, -> 1536 7.4, 9.3; but 16384 -> 2048, 16 tiles, 19.4, 15.0).  No more than
// 36 clusters of four run at once: 30 rows of 1243 in 36 tiles 7.1, in 37 or 38 12.7.
int int8_tile_split(int64_t tiles, int K, int nt, bool swap) {
  const int steps = (K + 63) / 64, most = swap ? nt / 32 : 4;
  int split = 1;
  while (split < most && tiles * (2 * split) <= sm_count() && steps >= 8 * split) split *= 2;
  if (!swap && split == 4 && tiles <= kFewTiles && steps >= 32) split = 8;
  return split;
}

cudaError_t launch_int8_tile(const Int8Args& all, void* workspace, cudaStream_t st, int expire, int nt, bool swap) {
  const int64_t slab = swap ? all.n : kTileSlab;
  for (int64_t off = 0; off < all.n; off += slab) {
    Int8Args A = off ? rest_of(all, off) : all;
    A.n = std::min(A.n, slab);
    if (swap) {
      A.n = all.N;
      A.N = (int32_t)all.n;
      std::swap(A.a, A.w);
      std::swap(A.lda, A.ldw);
      std::swap(A.a_scale, A.w_scale);
      A.swapped = 1;
    }
    const int split = int8_tile_split((int64_t)((A.N + CM - 1) / CM) * ((A.n + nt - 1) / nt), A.K, nt, swap);
    cudaError_t e = cudaSuccess;
    if (workspace && (e = launch_int8_expand_rows(A, workspace, st)) != cudaSuccess) return e;
    const uint8_t* ablocks = static_cast<const uint8_t*>(workspace);
    const bool wide = operand_align_w(A) == 16 && (workspace || operand_align(A) == 16);
    e = wide ? launch_rows<16>(A, ablocks, nt, split, expire, st) : launch_rows<1>(A, ablocks, nt, split, expire, st);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace bk
