// kern_int8_tile.cu -- the 8-bit product on the tensor cores, tiles of one CTA.
//
// tcgen05 has no 8-bit integer kind on sm_103a.  A code is exact in fp16, the product
// of two is an integer of at most 2^14, and fp32 holds every partial sum of 1024 of
// them exactly (2^24), so kind::f16 gives S exactly if the accumulators are taken
// to int32 every 1024 k at most.  They are double-buffered in tensor memory: one
// chunk's sums are added to int32 registers while the next chunk's MMAs run.
//
// A CTA computes 128 channels (MMA M; lanes of tensor memory) x NT rows (MMA N) over
// its share of K; the CTAs of a cluster share K, and add their int32 sums through
// distributed shared memory in a fixed order (integers: any order gives the same).
// Channels on M: a narrow batch costs narrow MMAs, and a warp's lanes hold 32
// neighbouring channels of a row, as the output wants them.  Warps of a CTA:
//   - 16 workers in four groups that take the k-steps (64 codes of every row) in turn: a
//     warp copies its rows' codes kDeep turns ahead (asynchronous copies to a ring of
//     its own: more in flight than registers allow), turns them into fp16 (128B
//     swizzle) and arrives on "full"; between them the workers drain finished chunks;
//   - two warps issue the MMAs of even and odd k-steps, each into accumulators of its own
//     (one issuer's wait, fence, four MMAs and commit take 450 clocks, narrow ones' pace),
//     committing to "empty" per k-step and "done" per chunk.
// Every wait is bounded; if one expires the CTA's partial sums are made again on CUDA
// cores, so the output is always whole.
#include <algorithm>
#include <type_traits>

#include "int8_common.cuh"
#include "tc_common.cuh"

namespace bk {
namespace {

using namespace tc;
using namespace i8;

constexpr int CM = 128;                 // channels of a tile
constexpr int KS = 64;                  // codes of a k-step (a 128-byte row of fp16)
constexpr int kWorkers = 16;
constexpr int kIssuers = 2;
constexpr int kThreads = 32 * (kWorkers + kIssuers);
constexpr int kMaxSplit = 8;
constexpr int kGroups = 4;              // worker groups, each a k-step of its own
constexpr int kChunk = 16 * kIssuers;   // k-steps between drains: 1024 k per accumulator
constexpr int kSmemBytes = 225 * 1024;  // for stages and copies in flight
constexpr int64_t kMaxRows = 65535ll * 128;   // rows of a launch (the grid's y limit)

template <int NT, int kAlign> struct Cfg {
  static constexpr int kUnits = (CM + NT) / 32;                // 8-row units of a k-step per warp
  // a unit in the ring: 4 chunks of 16 codes per row, or 5 (int8_common.cuh)
  static constexpr int kUnitBytes = 8 * 16 * (kAlign == 16 ? 4 : 5);
  static constexpr int kTurnBytes = kWorkers * kUnits * kUnitBytes;
  static constexpr int kStageBytes = (CM + NT) * 128;
  static constexpr int stages(int deep) {
    return std::min(8, (kSmemBytes - deep * kTurnBytes) / kStageBytes) / kIssuers * kIssuers;
  }
  // Turns in flight, and stages: at least one per group, and a stage always the same
  // issuer's.  (A warp that waits for its stage's last use has seen the k-step kGroups +
  // kStages back consumed; with fewer stages that says nothing of the use before the last,
  // whose phase has the same parity.)
  static constexpr int kDeep = stages(3) >= kGroups ? 3 : (stages(2) >= kGroups ? 2 : 1);
  static constexpr int kRingBytes = kDeep * kTurnBytes;
  static constexpr int kStages = stages(kDeep);
  static constexpr int kTmemCols = NT <= 32 ? 128 : (NT <= 64 ? 256 : 512);
  static constexpr int kSumPitch = CM + 4;                     // int32 per row of the exchange
  static_assert(4 * kSumPitch * NT <= kStages * kStageBytes, "exchange fits the stages");
  static_assert(kStages >= kGroups && kStages <= kChunk, "a chunk is drained before the one after the next starts");
};

struct __align__(8) TileShared {
  unsigned long long full[8], empty[8];
  unsigned long long done[2], drained[2];
  unsigned long long left;
  uint32_t tmem_base;
  int failed, left_failed;
};

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ int4 ld_cluster(uint32_t addr, uint32_t rank) {
  int4 v;
  asm volatile("{\n .reg .b32 a;\n mapa.shared::cluster.u32 a, %4, %5;\n"
               " ld.shared::cluster.v4.s32 {%0, %1, %2, %3}, [a];\n}"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr), "r"(rank) : "memory");
  return v;
}

// Four neighbouring outputs of a row.
template <typename T>
__device__ __forceinline__ void store4(const Int8Args& A, int64_t i, int j, const int4& s, float sa, const float (&sw)[4],
                                       const float (&bias)[4], bool vec) {
  T* p = static_cast<T*>(A.out) + i * A.ldo + j;
  const int v[4] = {s.x, s.y, s.z, s.w};
  T y[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    if constexpr (std::is_same<T, int32_t>::value) {
      y[c] = v[c];
    } else {
      float f = scaled(v[c], sa, sw[c]);
      if (A.bias) f = __fadd_rn(f, bias[c]);
      y[c] = out_cast<T>(f);
    }
  }
  if (vec && j + 4 <= A.N) {
    if constexpr (sizeof(T) == 4) *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(y);
    else *reinterpret_cast<uint2*>(p) = *reinterpret_cast<const uint2*>(y);
  } else {
#pragma unroll
    for (int c = 0; c < 4; ++c)
      if (j + c < A.N) p[c] = y[c];
  }
}

template <int NT, int kAlign>
__global__ void __launch_bounds__(kThreads, 1) k_int8_tile(const Int8Args A, int split, int expire) {
  using C = Cfg<NT, kAlign>;
  constexpr int kStages = C::kStages, kUnits = C::kUnits, kDeep = C::kDeep;
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
  const int all = (A.K + KS - 1) / KS;
  const int first = (int)((int64_t)all * rank / split), steps = (int)((int64_t)all * (rank + 1) / split) - first;
  const int chunks = (steps + kChunk - 1) / kChunk;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&sh->full[s], kWorkers / kGroups);
      mbar_init(&sh->empty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&sh->done[b], kIssuers);
      mbar_init(&sh->drained[b], kWorkers);
    }
    mbar_init(&sh->left, kIssuers);
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
  // Unit u: rows 32 u + 8 q .. + 7 of the tile's CM weight and NT activation rows, a lane 16
  // codes of a row.
  const int grp = warp >> 2, q = warp & 3;
  const int r = 8 * q + (lane >> 2), c = lane & 3;
  if (warp < kWorkers && c == 0) {
    // the first turn's weights on their way to L2 while the launch before this one ends
    const int k = KS * (first + grp);
#pragma unroll
    for (int u = 0; u < CM / 32; ++u)
      if (j0 + r + 32 * u < A.N && k < A.K)
        asm volatile("prefetch.global.L2 [%0];" ::"l"(A.w + (int64_t)(j0 + r + 32 * u) * A.ldw + k));
  }
  pdl_wait();
  pdl_trigger();

  if (warp < kWorkers) {
    // ---------------- workers ----------------
    const int8_t* wrow = A.w + (int64_t)(j0 + r) * A.ldw;
    const int8_t* arow = A.a + (i0 + r) * A.lda;
    const int8_t* any = aligned16(A.w);
    const int64_t wstep = 32 * A.ldw, astep = 32 * A.lda;
    // 32 bytes of fp16 per lane: chunks 2 c and 2 c + 1 of the row, swizzled
    const uint32_t at = smem_u32(base) + 128u * (uint32_t)r + ((32u * (uint32_t)c) ^ (16u * (uint32_t)(r & 7)));
    const uint32_t mine = smem_u32(ring) + (uint32_t)(warp * kDeep * kUnits * C::kUnitBytes) +
                          (uint32_t)((lane >> 2) * (C::kUnitBytes / 8) + 16 * c);
    auto copy = [&](int ks, int slot) {
      if (ks < steps) {
        const int k = KS * (first + ks) + 16 * c;
        uint32_t to = mine + (uint32_t)(slot * kUnits * C::kUnitBytes);
        const int8_t* row = wrow;
#pragma unroll
        for (int u = 0; u < kUnits; ++u, to += C::kUnitBytes) {
          if (u == CM / 32) row = arow;
          const bool live = u < CM / 32 ? j0 + r + 32 * u < A.N : i0 + r + 32 * (u - CM / 32) < A.n;
          const int shift = row_shift<kAlign>(row);
          copy_chunk(to, row, shift, k, live ? A.K : -16, any);
          if (kAlign != 16 && c == 0) copy_chunk(to + 64, row, shift, k + 64, live ? A.K : -16, any);
          row += u < CM / 32 ? wstep : astep;
        }
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int d = 0; d < kDeep; ++d) copy(grp + kGroups * d, d);
    constexpr int kCols = NT / 4;   // accumulator columns of this warp
    int acc[kCols];
#pragma unroll
    for (int e = 0; e < kCols; ++e) acc[e] = 0;
    const uint32_t tacc = tmem + ((uint32_t)(32 * (warp & 3)) << 16) + (uint32_t)(kCols * (warp >> 2));
    int drained = 0;   // chunks added to acc
    bool ok = true;
    auto drain = [&]() {
      const int b = drained & 1;
      ok = __all_sync(kFull, mbar_wait(&sh->done[b], (uint32_t)(drained >> 1) & 1u, failed));
      if (!ok) return;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      // (the odd k-steps' accumulator has nothing in a chunk of one)
      const int both = min(kIssuers, steps - drained * kChunk);
#pragma unroll 1
      for (int m = 0; m < both; ++m)
#pragma unroll
        for (int e = 0; e < kCols; e += 8) {
          uint32_t v[8];
          tmem_load8(v, tacc + (uint32_t)((kIssuers * b + m) * NT + e));
#pragma unroll
          for (int x = 0; x < 8; ++x) acc[e + x] += __float2int_rn(__uint_as_float(v[x]));
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
      const uint32_t to = at + s * (uint32_t)C::kStageBytes;
      if (kAlign != 16) __syncwarp();   // (chunks that other lanes copied)
      const uint32_t from = mine + (uint32_t)(slot * kUnits * C::kUnitBytes);
      constexpr int kBatch = 4;   // units whose loads are in flight together
#pragma unroll
      for (int u0 = 0; u0 < kUnits; u0 += kBatch) {
        uint32_t v[kBatch][4], h[4];
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
          if (u0 + u < kUnits) lds_chunk(v[u], from + (uint32_t)((u0 + u) * C::kUnitBytes));
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
          if (u0 + u < kUnits) {
            if constexpr (kAlign != 16) {
              uint32_t lo[4], hi[4];
#pragma unroll
              for (int i = 0; i < 4; ++i) lo[i] = v[u][i];
              lds_chunk(hi, from + (uint32_t)((u0 + u) * C::kUnitBytes) + 16u);
              merge16(v[u], lo, hi,
                      row_shift<kAlign>(u0 + u < CM / 32 ? wrow + (u0 + u) * wstep : arow + (u0 + u - CM / 32) * astep));
            }
            const uint32_t dst = to + 4096u * (uint32_t)(u0 + u);
            codes_f16(v[u][0], h[0], h[1]);
            codes_f16(v[u][1], h[2], h[3]);
            sts128(dst, h);
            codes_f16(v[u][2], h[0], h[1]);
            codes_f16(v[u][3], h[2], h[3]);
            sts128(dst ^ 16u, h);
          }
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh->full[s]);
      copy(ks + kGroups * kDeep, slot);
      if (++slot == kDeep) slot = 0;
      s += kGroups;
      wrap();
    }
    asm volatile("cp.async.wait_all;" ::: "memory");   // no copy outlives its thread
    while (ok && drained < chunks) drain();
    if (expire && threadIdx.x == 0) *failed = 1;
    // every MMA has completed: the sums go where the stages were
    if (ok) {
      int* to = reinterpret_cast<int*>(base) + 32 * (warp & 3) + lane;
#pragma unroll
      for (int e = 0; e < kCols; ++e) to[(kCols * (warp >> 2) + e) * C::kSumPitch] = acc[e];
    }
  } else {
    // ---------------- MMA issuers ----------------
    const int m = warp - kWorkers;
    const bool lead = elect_one();
    const uint32_t d = uniform(tmem) + (uint32_t)(m * NT);
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
        // the workers' stores, acquired above, before the MMAs' reads
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint64_t ad = desc0 + (uint64_t)(s * (uint32_t)(C::kStageBytes >> 4));
        const uint64_t bd = ad + (uint64_t)(CM * 128 >> 4);
        if (lead) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            mma_f16(d + (uint32_t)(kIssuers * b * NT), ad + 2 * e, bd + 2 * e, kIdesc, e > 0 ? 1u : accumulate);
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
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  if (warp == kWorkers)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(C::kTmemCols) : "memory");
  int* sums = reinterpret_cast<int*>(base);
  if (*failed) {
    // partial sums of this CTA's k range on CUDA cores
    const int k0 = KS * first, k1 = min(A.K, KS * (first + steps));
    for (int e = threadIdx.x; e < CM * NT; e += kThreads) {
      const int j = e % CM, i = e / CM;
      const int sum = j0 + j < A.N && i0 + i < A.n ? plain_sum(A, i0 + i, j0 + j, k0, k1) : 0;
      sums[i * C::kSumPitch + j] = sum;
    }
    __syncthreads();
  }
  if (split > 1) cluster_sync();

  // ---------------- output: rows rank, rank + split, ..., a warp per row ----------------
  const int j = j0 + 4 * lane;
  float sw[4], bias[4];
  int thr[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const bool in = j + c < A.N;
    sw[c] = in && A.w_scale ? A.w_scale[j + c] : 1.0f;
    bias[c] = in && A.bias ? A.bias[j + c] : 0.0f;
    thr[c] = in && A.thr ? A.thr[j + c] : 0;
  }
  const int size = A.type == BMLP_F32 || A.type == BMLP_I32 ? 4 : 2;
  const bool vec = ((reinterpret_cast<uintptr_t>(A.out) | (uintptr_t)(A.ldo * size)) & (uintptr_t)(4 * size - 1)) == 0;
  const int nw32 = 2 * ((A.N + 63) / 64);
  for (int t = (int)rank + split * warp; t < NT; t += split * (kWorkers + kIssuers)) {
    const int64_t i = i0 + t;
    if (i >= A.n) break;
    const uint32_t src = smem_u32(sums) + 4u * (uint32_t)(t * C::kSumPitch + 4 * lane);
    int4 v;
    if (split == 1) {
      v = *reinterpret_cast<const int4*>(sums + t * C::kSumPitch + 4 * lane);
    } else {
      int4 p[kMaxSplit];
#pragma unroll
      for (int q = 0; q < kMaxSplit; ++q)
        if (q < split) p[q] = ld_cluster(src, (uint32_t)q);
      v = p[0];
#pragma unroll
      for (int q = 1; q < kMaxSplit; ++q)
        if (q < split) {
          v.x += p[q].x; v.y += p[q].y; v.z += p[q].z; v.w += p[q].w;
        }
    }
    if (A.words) {
      uint32_t bits = 0u;
      bits |= (j + 0 < A.N && v.x >= thr[0]) ? 1u : 0u;
      bits |= (j + 1 < A.N && v.y >= thr[1]) ? 2u : 0u;
      bits |= (j + 2 < A.N && v.z >= thr[2]) ? 4u : 0u;
      bits |= (j + 3 < A.N && v.w >= thr[3]) ? 8u : 0u;
      bits <<= 4 * (lane & 7);
#pragma unroll
      for (int o = 1; o < 8; o <<= 1) bits |= __shfl_xor_sync(kFull, bits, o);
      const int word = j0 / 32 + (lane >> 3);
      if ((lane & 7) == 0 && word < nw32) reinterpret_cast<uint32_t*>(A.words)[i * nw32 + word] = bits;
    } else {
      const float sa = A.a_scale ? A.a_scale[i] : 1.0f;
      switch (A.type) {
        case BMLP_F32: store4<float>(A, i, j, v, sa, sw, bias, vec); break;
        case BMLP_F16: store4<__half>(A, i, j, v, sa, sw, bias, vec); break;
        case BMLP_BF16: store4<__nv_bfloat16>(A, i, j, v, sa, sw, bias, vec); break;
        default: store4<int32_t>(A, i, j, v, sa, sw, bias, vec);
      }
    }
  }
  if (split > 1) cluster_sync();   // no CTA leaves while its sums are read
}

template <int NT, int kAlign>
cudaError_t launch_tile(const Int8Args& A, int split, int expire, cudaStream_t st) {
  using C = Cfg<NT, kAlign>;
  constexpr int kSmem = 1024 + C::kStages * C::kStageBytes + C::kRingBytes + (int)sizeof(TileShared);
  const cudaError_t e = cudaFuncSetAttribute(k_int8_tile<NT, kAlign>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((A.N + CM - 1) / CM * split), (unsigned)((A.n + NT - 1) / NT));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kSmem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim = {(unsigned)split, 1u, 1u};
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, k_int8_tile<NT, kAlign>, A, split, expire);
}

template <int kAlign>
cudaError_t launch_rows(const Int8Args& A, int nt, int split, int expire, cudaStream_t st) {
  switch (nt) {
    case 32: return launch_tile<32, kAlign>(A, split, expire, st);
    case 64: return launch_tile<64, kAlign>(A, split, expire, st);
    case 96: return launch_tile<96, kAlign>(A, split, expire, st);
    default: return launch_tile<128, kAlign>(A, split, expire, st);
  }
}

}  // namespace

cudaError_t launch_int8_tile(const Int8Args& all, cudaStream_t st, int expire) {
  Int8Args A = all;
  A.n = std::min<int64_t>(all.n, kMaxRows);
  const int nt = A.n <= 32 ? 32 : (A.n <= 64 ? 64 : (A.n <= 96 ? 96 : 128));
  const int64_t tiles = (int64_t)((A.N + CM - 1) / CM) * ((A.n + nt - 1) / nt);
  const int steps = (A.K + KS - 1) / KS;
  int split = 1;
  while (split < kMaxSplit && tiles * (split + 1) <= sm_count() && steps >= 4 * (split + 1)) ++split;
  const cudaError_t e =
      operand_align(A) == 16 ? launch_rows<16>(A, nt, split, expire, st) : launch_rows<1>(A, nt, split, expire, st);
  if (e != cudaSuccess || all.n <= kMaxRows) return e;
  return launch_int8_tile(rest_of(all, kMaxRows), st, expire);
}

}  // namespace bk
