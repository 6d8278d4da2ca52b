// kern_int8_pair.cu -- the 8-bit product of many rows: both operands turned into fp16
// once, in the caller's workspace, then 256 x 256 tiles by pairs of CTAs.
//
// k_int8_expand writes an operand as blocks of 128 rows x 64 k of fp16, 16 KB each in
// the 128B-swizzled order that the MMAs read from shared memory, so a block is one
// linear copy; rows and codes past the operand's ends are zeros, and any stride and
// alignment ends here.  (Codes and sums are exact: kern_int8_tile.cu.)
//
// k_int8_pair: a cluster of two CTAs computes 256 channels (MMA M) x 256 rows (N) with
// tcgen05.mma.cta_group::2.  CTA r of the pair copies channels 128 r .. + 127 and rows
// 128 r .. + 127 of a k-step, 32 KB, in 512 clocks of MMA; its tensor memory receives
// the sums of its channels and all 256 rows, double-buffered in chunks of 1,024 k.
// The grid is persistent, a pair per two SMs.  Warps of a CTA (12, so that each may hold
// 168 registers):
//   - 8 epilogue warps add a finished chunk's sums to 128 int32 registers per thread (a
//     lane per channel) and, after a tile's last chunk, write its outputs;
//   - one thread copies blocks into a ring of kStages; both CTAs' copies complete on the
//     even one's barriers (tensor copies of a CTA pair may: forwarding the odd CTA's
//     completions by a thread there cost 700 clocks of a k-step's round trip);
//   - on the even CTA one warp issues the MMAs.
// Measured, both operands' expansion included: 16384 x 8192 -> 8192 1.17 to 1.22 ms = 1,800 to
// 1,880 TFLOP/s, signs of 65536 x 4096 -> 8192 2.21 to 2.27 ms = 1,940 to 1,990 (bf16 by the
// library 1,946).  Up to K = 1024 the one chunk's sums go from tensor memory to the outputs
// in fp32 as they are read: 47,880 x 332 -> 14,928 signs 420 us (through int32 registers
// 665).  A k-step takes 520 clocks where its MMAs take 512 (with forwarded completions
// 730 to 790); a chunk's read-out takes 4,900 of the 8,200 of the next chunk's MMAs, a tile's
// stores 4,900 (one instance per output type: with the types told apart inside the unrolled
// stores 21,000).  The expansion of 16384 and 8192 rows
// of 8192 takes 161 us (3.8 TB/s), of rows of 8191 195.
// Every wait is bounded; if one expires the pair's tiles are made again on CUDA cores.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include <cuda.h>

#include "int8_common.cuh"
#include "tc_common.cuh"

namespace bk {
namespace {

using namespace tc;
using namespace i8;

constexpr int kBlockRows = 128, kBlockK = 64;
constexpr int kBlockBytes = kBlockRows * kBlockK * 2;
constexpr int TP = 256;                  // channels, and rows, of a tile
constexpr int kStages = 7;
constexpr int kStageBytes = 2 * kBlockBytes;
constexpr int kChunk = 16;               // k-steps per accumulator: 1024 k
constexpr int kEpiWarps = 8, kCopyWarp = 8, kMmaWarp = 9;
constexpr int kThreads = 32 * 12;        // (two warps idle: registers are handed out by fours)
constexpr int kBand = 8;                 // row tiles that the pairs walk side by side

struct __align__(8) PairShared {
  unsigned long long full[kStages], empty[kStages];
  unsigned long long done[2], drained[2];
  unsigned long long left;
  uint32_t tmem_base;
  int failed, left_failed;
};
constexpr int kSmem = 1024 + kStages * kStageBytes + (int)sizeof(PairShared);

// ---------------------------------------------------------------------------
// Operand to blocks: a warp takes 8 rows x 64 codes at a time (1 KB written).
// ---------------------------------------------------------------------------
struct ExpandArgs {
  const int8_t *x0, *x1;
  int64_t ld0, ld1, rows0, rows1;
  int64_t units0, units;      // 8-row strips of the first operand, of both
  uint8_t *blocks0, *blocks1;
  int32_t K, nkb;
};

constexpr int kExpandThreads = 256;

// kExpandSteps: blocks along k per warp and turn.
template <int kAlign, int kExpandSteps>
__global__ void __launch_bounds__(kExpandThreads) k_int8_expand(const ExpandArgs E) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, c = lane & 3;
  const int turns = (E.nkb + kExpandSteps - 1) / kExpandSteps;
  const int64_t total = E.units * turns;
  for (int64_t t = (int64_t)blockIdx.x * (kExpandThreads / 32) + (threadIdx.x >> 5); t < total;
       t += (int64_t)gridDim.x * (kExpandThreads / 32)) {
    int64_t strip = t / turns;
    const int kb0 = (int)(t % turns) * kExpandSteps;
    const bool second = strip >= E.units0;
    if (second) strip -= E.units0;
    const int64_t row = 8 * strip + (lane >> 2);
    const bool live = row < (second ? E.rows1 : E.rows0);
    const int8_t* src = (second ? E.x1 : E.x0) + (live ? row : 0) * (second ? E.ld1 : E.ld0);
    const int r = (int)(row & (kBlockRows - 1));
    uint8_t* to = (second ? E.blocks1 : E.blocks0) + (row / kBlockRows * E.nkb + kb0) * (int64_t)kBlockBytes + 128 * r +
                  ((32 * c) ^ (16 * (r & 7)));
    uint32_t v[kExpandSteps][4];
    const int shift = row_shift<kAlign>(src);
    if (live && kBlockK * (kb0 + kExpandSteps) + (kAlign == 16 ? 0 : 16) <= E.K) {
#pragma unroll
      for (int i = 0; i < kExpandSteps; ++i) load16_inside<kAlign>(v[i], src, shift, kBlockK * (kb0 + i) + 16 * c);
    } else {
#pragma unroll
      for (int i = 0; i < kExpandSteps; ++i)
        load16<kAlign>(v[i], src, shift, kBlockK * (kb0 + i) + 16 * c, live ? E.K : -16);
    }
#pragma unroll
    for (int i = 0; i < kExpandSteps; ++i) {
      if (kb0 + i < E.nkb) {
        uint32_t h[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) codes_f16(v[i][e], h[2 * e], h[2 * e + 1]);
        uint8_t* p = to + (int64_t)i * kBlockBytes;
        *reinterpret_cast<uint4*>(p) = make_uint4(h[0], h[1], h[2], h[3]);
        *reinterpret_cast<uint4*>(reinterpret_cast<uint8_t*>(reinterpret_cast<uintptr_t>(p) ^ 16)) =
            make_uint4(h[4], h[5], h[6], h[7]);
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Pairs
// ---------------------------------------------------------------------------
__device__ __forceinline__ uint32_t pair_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void pair_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Bounded wait with cluster-scope acquire (the barrier collects arrivals of the peer).
__device__ __forceinline__ bool mbar_wait_cluster(unsigned long long* bar, uint32_t parity, volatile int* failed) {
  const uint32_t a = smem_u32(bar);
  uint32_t ok;
  auto try_wait = [&]() {
    asm volatile(
        "{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n"
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
    if (clock64() - t0 > kWaitCycles) {
      *failed = 1;
      return false;
    }
  }
}

// Arrive on the barrier at the same offset in CTA 0 of the cluster.
__device__ __forceinline__ void mbar_arrive_rank0(unsigned long long* bar) {
  uint32_t remote;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(remote) : "r"(smem_u32(bar)));
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(remote) : "memory");
}

__device__ __forceinline__ void mma_f16_pair(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc,
                                             uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}"
      ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate));
}

// Arrive once on the barrier at this offset in both CTAs of the pair when the MMAs
// issued so far complete.
__device__ __forceinline__ void mma_commit_pair(unsigned long long* bar) {
  const uint16_t mask = 0x3;
  asm volatile(
      "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
      ::"r"(smem_u32(bar)), "h"(mask) : "memory");
}

// Tile t of ctiles x rtiles: bands of kBand row tiles, inside a band channel by channel.
__device__ __forceinline__ void tile_at(int64_t t, int ctiles, int64_t rtiles, int& ct, int64_t& rt) {
  const int64_t band = t / ((int64_t)kBand * ctiles);
  const int64_t first = band * kBand, wide = rtiles - first < kBand ? rtiles - first : kBand;
  const int64_t in = t - first * ctiles;
  ct = (int)(in / wide);
  rt = first + in % wide;
}

// Tensor copy of one block (128 rows of 64 from row y of the map) to this CTA's shared
// memory, completing on a barrier of either CTA of the pair.
__device__ __forceinline__ void copy_block(void* dst, const CUtensorMap* map, int y, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
      ::"r"(smem_u32(dst)), "l"(map), "r"(0), "r"(y), "r"(bar) : "memory");
}
// The barrier at this offset in CTA 0 of the cluster.
__device__ __forceinline__ uint32_t rank0_address(unsigned long long* bar) {
  uint32_t remote;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(remote) : "r"(smem_u32(bar)));
  return remote;
}

// What the kernel writes: one instance each, so that the unrolled stores stay short.
struct Signs {};
template <typename T> struct IsSigns { static constexpr bool value = false; };
template <> struct IsSigns<Signs> { static constexpr bool value = true; };

// Bit e of lane l's word to bit l of lane e's.
__device__ __forceinline__ uint32_t transpose_bits(uint32_t x) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int s = 16; s > 0; s >>= 1) {
    const uint32_t low = s == 16 ? 0x0000FFFFu : (s == 8 ? 0x00FF00FFu : (s == 4 ? 0x0F0F0F0Fu : (s == 2 ? 0x33333333u : 0x55555555u)));
    const uint32_t y = __shfl_xor_sync(kFull, x, s);
    x = lane & s ? (x & ~low) | ((y >> s) & low) : (x & low) | ((y << s) & ~low);
  }
  return x;
}

// A warp's outputs of 32 rows from i on (`rows` of them some), 32 channels from jw on, a lane per
// channel; V: int32 sums, or the same as fp32 where they are exact.
template <typename TOut, typename V>
__device__ __forceinline__ void put_group(const Int8Args& A, const V (&v)[32], int64_t i, int rows, int jw, float sw,
                                          float bias, V thr) {
  const int lane = threadIdx.x & 31, j = jw + lane;
  if constexpr (IsSigns<TOut>::value) {
    const int nw32 = 2 * ((A.N + 63) / 64);
    uint32_t bits = 0u;
#pragma unroll
    for (int e = 0; e < 32; ++e) bits |= v[e] >= thr ? 1u << e : 0u;
    bits = transpose_bits(j < A.N ? bits : 0u);
    if (lane < rows && (jw >> 5) < nw32) reinterpret_cast<uint32_t*>(A.words)[(i + lane) * nw32 + (jw >> 5)] = bits;
  } else {
    TOut* to = static_cast<TOut*>(A.out) + i * A.ldo + j;
    const bool has_bias = A.bias != nullptr;
    const float sal = A.a_scale && lane < rows ? A.a_scale[i + lane] : 1.0f;
#pragma unroll
    for (int e = 0; e < 32; ++e, to += A.ldo) {
      const float sa = __shfl_sync(kFull, sal, e);
      TOut y;
      if constexpr (std::is_same<TOut, int32_t>::value) {
        y = (int32_t)v[e];
      } else {
        const float f = scaled((float)v[e], sa, sw);
        y = out_cast<TOut>(has_bias ? __fadd_rn(f, bias) : f);
      }
      if (e < rows && j < A.N) *to = y;
    }
  }
}

template <typename TOut>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
    k_int8_pair(const Int8Args A, const __grid_constant__ CUtensorMap wmap, const __grid_constant__ CUtensorMap amap,
                int nkb, int ctiles, int64_t rtiles, int expire) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  PairShared* sh = reinterpret_cast<PairShared*>(base + kStages * kStageBytes);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = pair_rank();
  const int64_t pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  const int64_t tiles = (int64_t)ctiles * rtiles;
  const int chunks = (nkb + kChunk - 1) / kChunk;
  volatile int* failed = &sh->failed;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&sh->full[s], 1);
      mbar_init(&sh->empty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&sh->done[b], 1);
      mbar_init(&sh->drained[b], 2 * kEpiWarps);
    }
    mbar_init(&sh->left, 1);
    sh->failed = sh->left_failed = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;"
                 ::"r"(smem_u32(&sh->tmem_base)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  pair_sync();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = sh->tmem_base;
  pdl_wait();
  pdl_trigger();

  if (warp < kEpiWarps) {
    // ---------------- epilogue ----------------
    const int quarter = warp & 3, half = warp >> 2;   // 32 channels; 128 of the tile's rows
    const uint32_t tacc = tmem + ((uint32_t)(32 * quarter) << 16) + (uint32_t)(128 * half);
    uint32_t seen = 0;   // chunks drained
    bool ok = true;
#pragma unroll 1
    for (int64_t t = pair; t < tiles && ok; t += pairs) {
      int ct;
      int64_t rt;
      tile_at(t, ctiles, rtiles, ct, rt);
      const int jw = TP * ct + 128 * (int)rank + 32 * quarter, j = jw + lane;
      const int64_t i0 = TP * rt + 128 * half;
      const float sw = j < A.N && A.w_scale ? A.w_scale[j] : 1.0f;
      const float bias = j < A.N && A.bias ? A.bias[j] : 0.0f;
      const int thr = j < A.N && A.thr ? A.thr[j] : 0;
      const int rows = (int)max((int64_t)0, min((int64_t)128, A.n - i0));
      if (chunks == 1) {
        // one chunk: the sums are in fp32 exactly, and go out as they are read
        const uint32_t b = seen & 1u;
        ok = __all_sync(kFull, mbar_wait_cluster(&sh->done[b], (seen >> 1) & 1u, failed));
        if (!ok || expire) break;
        ++seen;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        // (a threshold that no sum reaches, or every one, as an infinity: others are exact in fp32)
        const float thrf = thr > 1 << 24 ? INFINITY : (thr < -(1 << 24) ? -INFINITY : (float)thr);
        // (all are read before the arrival and stored after it, since its release waits for stores under
        // way: 37,155 x 55 -> 13,908 signs 242 us, read and stored by quarters 290)
        uint32_t v[8][16];
#pragma unroll
        for (int e = 0; e < 8; ++e) tmem_load16(v[e], tacc + 256u * b + 16u * (uint32_t)e);
#pragma unroll
        for (int e = 0; e < 8; ++e) tmem_wait_ld(v[e]);
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive_rank0(&sh->drained[b]);
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          float f[32];
#pragma unroll
          for (int e = 0; e < 32; ++e) f[e] = __uint_as_float(v[2 * g + (e >> 4)][e & 15]);
          put_group<TOut>(A, f, i0 + 32 * g, rows - 32 * g, jw, sw, bias, thrf);
        }
        continue;
      }
      int acc[128];
#pragma unroll
      for (int e = 0; e < 128; ++e) acc[e] = 0;
#pragma unroll 1
      for (int ch = 0; ch < chunks; ++ch, ++seen) {
        const uint32_t b = seen & 1u;
        ok = __all_sync(kFull, mbar_wait_cluster(&sh->done[b], (seen >> 1) & 1u, failed));
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
        for (int e = 0; e < 128; e += 16) {
          uint32_t v[16];
          tmem_load16(v, tacc + 256u * b + (uint32_t)e);
          tmem_wait_ld(v);
#pragma unroll
          for (int x = 0; x < 16; ++x) acc[e + x] += __float2int_rn(__uint_as_float(v[x]));
        }
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive_rank0(&sh->drained[b]);
      }
      if (!ok || expire) break;
#pragma unroll
      for (int g = 0; g < 4; ++g)
        put_group<TOut>(A, *reinterpret_cast<const int(*)[32]>(acc + 32 * g), i0 + 32 * g, rows - 32 * g, jw, sw, bias, thr);
    }
    if (expire && threadIdx.x == 0) *failed = 1;
  } else if (warp == kCopyWarp) {
    // ---------------- copies ----------------
    if (lane == 0) {
      uint32_t s = 0, ph = 1;
      int64_t copied = 0;
      bool ok = true;
#pragma unroll 1
      for (int64_t t = pair; t < tiles && ok; t += pairs) {
        int ct;
        int64_t rt;
        tile_at(t, ctiles, rtiles, ct, rt);
        const int wy = (2 * ct + (int)rank) * nkb * kBlockRows, ay = (int)((2 * rt + rank) * nkb * kBlockRows);
#pragma unroll 1
        for (int ks = 0; ks < nkb; ++ks) {
          ok = mbar_wait(&sh->empty[s], ph, failed);
          if (!ok) break;
          uint8_t* to = base + s * kStageBytes;
          if (rank == 0) mbar_arrive_tx(&sh->full[s], 2 * kStageBytes);
          const uint32_t bar = rank0_address(&sh->full[s]);
          copy_block(to, &wmap, wy + ks * kBlockRows, bar);
          copy_block(to + kBlockBytes, &amap, ay + ks * kBlockRows, bar);
          ++copied;
          if (++s == kStages) {
            s = 0;
            ph ^= 1u;
          }
        }
      }
      if (!ok && rank == 0) {
        // no copy outlives its CTA: the last phases hold both CTAs' copies (where the odd one
        // stopped earlier, the wait's limit is time enough for what is in flight)
        for (int64_t k = copied > kStages ? copied - kStages : 0; k < copied; ++k)
          mbar_wait(&sh->full[k % kStages], (uint32_t)(k / kStages) & 1u, &sh->left_failed, 2000000ull);
      }
    }
  } else if (rank == 0 && warp == kMmaWarp) {
    // ---------------- MMA issuer of the pair ----------------
    const bool lead = elect_one();
    const uint32_t d = uniform(tmem);
    const uint64_t desc0 = smem_desc(uniform(smem_u32(base)));
    constexpr uint32_t kIdesc = idesc_f16(TP, TP);
    uint32_t s = 0, ph = 0, made = 0;   // chunks issued
    bool ok = true;
#pragma unroll 1
    for (int64_t t = pair; t < tiles && ok; t += pairs) {
#pragma unroll 1
      for (int ch = 0; ch < chunks && ok; ++ch, ++made) {
        const uint32_t b = made & 1u;
        ok = __all_sync(kFull, mbar_wait_cluster(&sh->drained[b], ((made >> 1) & 1u) ^ 1u, failed));
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const int end = min(nkb, (ch + 1) * kChunk);
#pragma unroll 1
        for (int ks = ch * kChunk; ks < end; ++ks) {
          ok = __all_sync(kFull, mbar_wait_cluster(&sh->full[s], ph, failed));
          if (!ok) break;
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const uint64_t ad = desc0 + (uint64_t)(s * (uint32_t)(kStageBytes >> 4));
          const uint64_t bd = ad + (uint64_t)(kBlockBytes >> 4);
          if (lead) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              mma_f16_pair(d + 256u * b, ad + 2 * e, bd + 2 * e, kIdesc, (ks > ch * kChunk || e > 0) ? 1u : 0u);
            mma_commit_pair(&sh->empty[s]);
          }
          if (++s == kStages) {
            s = 0;
            ph ^= 1u;
          }
        }
        if (ok && lead) mma_commit_pair(&sh->done[b]);
        __syncwarp();
      }
    }
    if (lead) {
      // no MMA outlives its operands and its tensor memory
      mma_commit_pair(&sh->left);
      mbar_wait(&sh->left, 0, &sh->left_failed);
    }
    __syncwarp();
  }
  __syncwarp();
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  pair_sync();   // no CTA releases TMEM or leaves while its peer may still use the pair
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  if (warp == kMmaWarp)
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
  // did a wait of either CTA expire?
  uint32_t peer;
  asm volatile("{\n .reg .b32 a;\n mapa.shared::cluster.u32 a, %1, %2;\n ld.shared::cluster.u32 %0, [a];\n}"
               : "=r"(peer) : "r"(smem_u32(&sh->failed)), "r"(rank ^ 1u) : "memory");
  const bool redo = peer != 0u || *failed != 0;
  // the last arrival that the even CTA's commits send here
  if (rank != 0 && threadIdx.x == 0) mbar_wait(&sh->left, 0, &sh->left_failed);
  __syncwarp();
  pair_sync();
  if (redo) {
    for (int64_t t = pair; t < tiles; t += pairs) {
      int ct;
      int64_t rt;
      tile_at(t, ctiles, rtiles, ct, rt);
      plain_tile(A, TP * rt, TP, TP * ct + 128 * (int)rank, 128);
    }
  }
}

template <int kAlign, int kSteps>
cudaError_t expand(const ExpandArgs& E, cudaStream_t st) {
  const int64_t turns = E.units * ((E.nkb + kSteps - 1) / kSteps);
  const int64_t ctas = (turns + kExpandThreads / 32 - 1) / (kExpandThreads / 32);
  return launch_kernel(k_int8_expand<kAlign, kSteps>, dim3((unsigned)std::min<int64_t>(ctas, 8ll * sm_count())),
                       dim3(kExpandThreads), 0, st, true, E);
}

int64_t padded(int64_t rows) { return (rows + TP - 1) / TP * TP; }
int64_t row_bytes(int K) { return (int64_t)((K + kBlockK - 1) / kBlockK) * kBlockK * 2; }

}  // namespace

int64_t int8_rows_workspace(int64_t n, int K) {
  n = std::min(n, kTileSlab);
  return row_bytes(K) * ((n + kBlockRows - 1) / kBlockRows * kBlockRows);
}

cudaError_t launch_int8_expand_rows(const Int8Args& A, void* workspace, cudaStream_t st) {
  ExpandArgs E = {};
  E.x1 = A.a;
  E.ld1 = A.lda;
  E.rows1 = A.n;
  E.units = (A.n + 7) / 8;   // (what the last block's other rows hold is dropped)
  E.blocks1 = static_cast<uint8_t*>(workspace);
  E.K = A.K;
  E.nkb = (A.K + kBlockK - 1) / kBlockK;
  const bool wide = ((reinterpret_cast<uintptr_t>(A.a) | (A.n > 1 ? (uintptr_t)A.lda : 0)) & 15) == 0;
  return wide ? expand<16, 1>(E, st) : expand<1, 1>(E, st);
}

int64_t int8_pair_workspace(int64_t n, int K, int64_t N) {
  return row_bytes(K) * (padded(N) + std::min(padded(n), kPairSlab));
}

namespace {

// Map of an operand's blocks: rows of 64 fp16 (already in the order that shared memory
// holds), 128 at a time.
bool block_map(CUtensorMap* map, void* blocks, int64_t rows) {
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
  if (!encode) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)kBlockK, (cuuint64_t)rows}, strides[1] = {2 * kBlockK};
  const cuuint32_t box[2] = {kBlockK, kBlockRows}, steps[2] = {1, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, blocks, dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) ==
         CUDA_SUCCESS;
}

template <typename TOut>
cudaError_t launch_out(const Int8Args& A, const CUtensorMap& wmap, const CUtensorMap& amap, int nkb, cudaStream_t st,
                       int expire) {
  static std::atomic<uint64_t> done{0};
  const cudaError_t e = allow_smem(done, k_int8_pair<TOut>, kSmem);
  if (e != cudaSuccess) return e;
  const int ctiles = (int)(padded(A.N) / TP);
  const int64_t rtiles = padded(A.n) / TP;
  const int64_t pairs = std::min<int64_t>(sm_count() / 2, (int64_t)ctiles * rtiles);
  return launch_kernel(k_int8_pair<TOut>, dim3((unsigned)(2 * pairs)), dim3(kThreads), (size_t)kSmem, st, true, A, wmap,
                       amap, nkb, ctiles, rtiles, expire);
}

}  // namespace

cudaError_t launch_int8_pair(const Int8Args& all, void* workspace, cudaStream_t st, int expire) {
  const int nkb = (all.K + kBlockK - 1) / kBlockK;
  uint8_t* wblocks = static_cast<uint8_t*>(workspace);
  uint8_t* ablocks = wblocks + row_bytes(all.K) * padded(all.N);
  const bool wide = operand_align(all) == 16;
  for (int64_t off = 0; off < all.n; off += kPairSlab) {
    Int8Args A = off ? rest_of(all, off) : all;
    A.n = std::min(A.n, kPairSlab);
    ExpandArgs E = {};
    E.x0 = A.w; E.x1 = A.a;
    E.ld0 = A.ldw; E.ld1 = A.lda;
    E.rows0 = A.N; E.rows1 = A.n;
    E.units0 = off ? 0 : padded(A.N) / 8;   // the channels once
    E.units = E.units0 + padded(A.n) / 8;
    E.blocks0 = wblocks; E.blocks1 = ablocks;
    E.K = A.K; E.nkb = nkb;
    CUtensorMap wmap, amap;
    if (!block_map(&wmap, wblocks, padded(A.N) * nkb) || !block_map(&amap, ablocks, padded(A.n) * nkb))
      return cudaErrorNotSupported;
    cudaError_t e = wide ? expand<16, 4>(E, st) : expand<1, 4>(E, st);
    if (e != cudaSuccess) return e;
    if (A.words) e = launch_out<Signs>(A, wmap, amap, nkb, st, expire);
    else if (A.type == BMLP_F32) e = launch_out<float>(A, wmap, amap, nkb, st, expire);
    else if (A.type == BMLP_F16) e = launch_out<__half>(A, wmap, amap, nkb, st, expire);
    else if (A.type == BMLP_BF16) e = launch_out<__nv_bfloat16>(A, wmap, amap, nkb, st, expire);
    else e = launch_out<int32_t>(A, wmap, amap, nkb, st, expire);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace bk
