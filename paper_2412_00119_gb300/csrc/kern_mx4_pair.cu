// kern_mx4_pair.cu -- the microscaled 4-bit product of many rows: 256 x 256 tiles by pairs of CTAs,
// for operands that tensor copies can take (kern_mx4_tile.cu has the formats in shared and
// tensor memory).
//
// A cluster of two CTAs computes 256 channels (MMA M) x up to 256 rows (N, as many as the tile
// has, up to 32) with tcgen05.mma.cta_group::2.  CTA r copies channels 128 r .. + 127 and the r-th half
// of the rows: 32 KB per 256 codes, in 512 clocks of MMA; its tensor memory receives the sums of
// its channels and all rows, and it needs the scales of its channels and of all rows there.
// The grid is persistent, a pair per two SMs.  Two accumulators of 256 columns and the scales
// do not fit tensor memory side by side: the accumulators share 128 columns, which the epilogue
// reads first.  Warps of a CTA: 16 write outputs, four bring scales to a ring in shared memory, four
// take them from there to tensor memory, one thread copies codes (both CTAs' copies complete on the
// even one's barriers), and on the even CTA one warp issues the MMAs.
// What a CTA tells the other of is tensor copies, which complete on the even CTA's barriers, and tensor
// memory, in the order of tcgen05's fences.  The scales go there by tcgen05.st, since a tcgen05.cp that the even CTA
// issues reads what the odd one's threads have stored to its shared memory, and that needs a release for the
// cluster: 16384 x 8192 -> 8192 439 us with one for each step (435 to 450 with the cells in a ring of their own).
// Measured: 16384 x 8192 -> 8192 366 to 401 us (5.5 to 6.0 PFLOP/s), 4096 x 4096 -> 4096 35.5, 16384 x 4096 -> 4096 by 16
// groups 114 to 129.  Bound: the scales' way.  A step takes 870 clocks, its MMAs 512: the MMA warp waits 350 for
// scales and 170 for codes (an SM takes in a step's 32 KB in 600); the warps that take scales to tensor memory wait
// 310 for the MMAs of five steps before, and are busy else.
// Every wait is bounded; if one expires the pair's tiles are made again on CUDA cores.
#include <algorithm>

#include "mx4_common.cuh"

namespace bk {
namespace {

using namespace tc;
using namespace mx4;

constexpr int TP = 256;                  // channels, and rows at most, of a tile
constexpr int kStepBytes = 128;          // of a row per stage: 256 codes
constexpr int kBlockBytes = 128 * kStepBytes;
constexpr int kStageBytes = 2 * kBlockBytes;
constexpr int kStages = 6;
constexpr int kUnit = 4;                 // steps whose scales are brought at once: 32 bytes of a row
constexpr int kUnits = 2;                // in the ring
constexpr int kCells = 6 * kCell, kUnitBytes = kUnit * kCells;   // of a step: two of the channels, four of the rows (two halves of 128, twice)
constexpr int kEpiWarps = 16, kScaleWarps = 4, kPutWarp = kEpiWarps + kScaleWarps, kMmaWarp = kPutWarp + 4, kCopyWarp = kMmaWarp + 1;
constexpr int kThreads = 32 * (kCopyWarp + 1);
constexpr int kShared = 128;             // columns of both accumulators
constexpr int kSfCol = 2 * TP - kShared; // scales: 24 columns a step
constexpr int kSlots = 5, kSlotCols = 24;
static_assert(kSfCol + kSlots * kSlotCols <= 512 && kStageBytes % 1024 == 0, "tensor memory, swizzle atoms");
static_assert(kPutWarp % 4 == 0 && kSlots < kStages, "a warp's lanes of tensor memory; every stage's MMAs are waited for");
constexpr int kBand = 8;                 // row tiles that the pairs walk side by side

struct __align__(8) PairShared {
  unsigned long long full[kStages], empty[kStages], scaled[kSlots];   // codes; read; scales in tensor memory
  unsigned long long loaded[kUnits], taken[kUnits];                  // scales in the ring; read
  unsigned long long done[2], drained;
  unsigned long long left;
  uint32_t tmem_base;
  int failed, left_failed;
};
constexpr int64_t pair_smem(int E) {
  return 1024 + (int64_t)kStages * kStageBytes + kUnits * kUnitBytes + (int64_t)sizeof(PairShared) + 8 * (int64_t)(E + 1);
}

__device__ __forceinline__ uint32_t pair_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void pair_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The barrier at this offset in CTA 0 of the cluster, and an arrival on it.
__device__ __forceinline__ uint32_t rank0_address(unsigned long long* bar) {
  uint32_t remote;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(remote) : "r"(smem_u32(bar)));
  return remote;
}
// It tells that columns of tensor memory are read or written: between tcgen05.fence::before_thread_sync here and
// ::after_thread_sync there it has to order execution alone, and releases no memory.
__device__ __forceinline__ void mbar_arrive_rank0(unsigned long long* bar) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(rank0_address(bar)) : "memory");
}

__device__ __forceinline__ void mma_mx4_pair(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t sfa,
                                             uint32_t sfb, uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %6, 0;\n"
      " tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n}"
      ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate));
}
// Four columns' words of a lane.
__device__ __forceinline__ void lds_cell(uint32_t* v, uint32_t a) {
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(a) : "memory");
}
// Words to 8 columns of this warp's lanes of tensor memory.
__device__ __forceinline__ void tmem_store8(uint32_t taddr, const uint32_t (&v)[8]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
      ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
}
// Arrive once on the barrier at this offset in both CTAs of the pair when what was issued so far completes.
__device__ __forceinline__ void mma_commit_pair(unsigned long long* bar) {
  const uint16_t mask = 0x3;
  asm volatile(
      "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
      ::"r"(smem_u32(bar)), "h"(mask) : "memory");
}
// Tensor copies to this CTA's shared memory, completing on a barrier of either CTA of the pair.
__device__ __forceinline__ void copy_w(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
      ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
__device__ __forceinline__ void copy_a(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
      ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}

// Tile t: bands of kBand row tiles, inside a band channel by channel.
__device__ __forceinline__ Item tile_at(const Items& I, int64_t t) {
  const int64_t per = (int64_t)kBand * I.ctiles;
  const int64_t band = (t | per) >> 31 == 0 ? (int64_t)((uint32_t)t / (uint32_t)per) : t / per;
  const int64_t left = I.rtiles - band * kBand;
  const uint32_t wide = left < kBand ? (uint32_t)left : (uint32_t)kBand;
  const int64_t in = t - band * per;
  const int64_t ct = in >> 31 == 0 ? (int64_t)((uint32_t)in / wide) : in / wide;
  return I.at(band * kBand + (in - ct * wide), TP * (int)ct);
}

template <typename TOut>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
    k_mx4_pair(const Mx4Args A, const __grid_constant__ Maps maps, int ctiles, int whole, int expire) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  PairShared* sh = reinterpret_cast<PairShared*>(base + kStages * kStageBytes + kUnits * kUnitBytes);
  int32_t* groups = reinterpret_cast<int32_t*>(sh + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = pair_rank();
  volatile int* failed = &sh->failed;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&sh->full[s], 1);
      mbar_init(&sh->empty[s], 1);
    }
    for (int s = 0; s < kSlots; ++s) mbar_init(&sh->scaled[s], 2 * 4);
    for (int u = 0; u < kUnits; ++u) {
      mbar_init(&sh->loaded[u], kScaleWarps);
      mbar_init(&sh->taken[u], 4);
    }
    for (int b = 0; b < 2; ++b) mbar_init(&sh->done[b], 1);
    mbar_init(&sh->drained, 2 * kEpiWarps);
    mbar_init(&sh->left, 1);
    sh->failed = sh->left_failed = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;"
                 ::"r"(smem_u32(&sh->tmem_base)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  if (warp == kCopyWarp && lane == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.w) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.a) : "memory");
  }
  pdl_wait();
  pdl_trigger();
  if (A.offsets && warp == 0) group_tiles(A, TP, groups);
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  pair_sync();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = sh->tmem_base;
  const Items items = {A.offsets ? groups : nullptr, A.offsets ? groups + A.E + 1 : nullptr, A.E, TP, ctiles, 0, 0,
                       A.offsets ? (int64_t)groups[A.E] : (A.n + TP - 1) / TP, A.n};
  const int64_t tiles = items.rtiles * ctiles, pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  const int64_t bytes = ((int64_t)A.K + 1) / 2;
  const int steps = (int)((bytes + kStepBytes - 1) / kStepBytes);

  if (warp < kEpiWarps) {
    // ---------------- outputs ----------------
    const int quarter = warp & 3, part = warp >> 2;   // blocks of 16 rows: part, part + 4, ..
    const bool has_rs = A.row_scale != nullptr, has_bias = A.bias != nullptr;
    uint32_t seen = 0;
    bool ok = true;
#pragma unroll 1
    for (int64_t t = pair; t < tiles && ok; t += pairs, ++seen) {
      const Item it = tile_at(items, t);
      const int j = it.j0 + 128 * (int)rank + 32 * quarter + lane;
      const bool live = j < A.N;
      // what the outputs need from memory, asked for before the sums are there
      const float bias = has_bias && live ? A.bias[it.e * A.ldb + j] : 0.0f;
      float rs[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int x = 16 * (4 * c + part) + (lane & 15);
        rs[c] = has_rs && x < it.rows ? A.row_scale[it.r0 + x] : 1.0f;
      }
      const uint32_t b = seen & 1u, tacc = tmem + ((uint32_t)(32 * quarter) << 16) + b * (uint32_t)(TP - kShared);
      ok = __all_sync(kFull, wait_phase<kOrder>(&sh->done[b], (seen >> 1) & 1u, failed));
      if (!ok) break;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      // the columns that the accumulators share: the second one's first eight blocks of 16, the first one's last
      static_assert(kShared == 128 && TP == 256, "blocks 0 to 7 and 8 to 15: two of each warp's");
      const int c0 = b ? 0 : 2;   // this warp's first of two
      uint32_t v[2][16];
#pragma unroll
      for (int i = 0; i < 2; ++i) tmem_load16(v[i], tacc + 16u * (uint32_t)(4 * (c0 + i) + part));
#pragma unroll
      for (int i = 0; i < 2; ++i) tmem_wait_ld(v[i]);
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive_rank0(&sh->drained);
      auto put = [&](const uint32_t (&f)[16], int c) {
        const int x0 = 16 * (4 * c + part), left = it.rows - x0;
        if (left <= 0 || expire) return;
        float by = rs[0];
#pragma unroll
        for (int i = 1; i < 4; ++i)
          if (c == i) by = rs[i];
        put_rows(static_cast<TOut*>(A.out) + (it.r0 + x0) * A.ldo + j, A.ldo, f, by, bias, left, live);
      };
#pragma unroll
      for (int i = 0; i < 2; ++i) put(v[i], c0 + i);
      // (read before the next tile's arrival: after that this accumulator may be written again)
#pragma unroll 1
      for (int i = 2; i < 4; ++i) {
        const int c = c0 ^ i;
        if (16 * (4 * c + part) >= it.rows) continue;
        uint32_t f[16];
        tmem_load16(f, tacc + 16u * (uint32_t)(4 * c + part));
        tmem_wait_ld(f);
        put(f, c);
      }
    }
    if (expire && threadIdx.x == 0) *failed = 1;
  } else if (warp < kPutWarp) {
    // ---------------- scales to the ring ----------------
    // A lane loads 32 bytes of its channel and of its row of each half, and stores them as cells of 128 rows x 128
    // codes: the four bytes of row r at 16 (r % 32) + 4 (r / 32).
    const int q = warp - kEpiWarps, r = 32 * q + lane;   // this lane's channel, and row of each half
    const int len = (int)(((int64_t)A.K + 31) / 32);
    const uint32_t ring = smem_u32(base) + (uint32_t)(kStages * kStageBytes) + 16u * (uint32_t)lane + 4u * (uint32_t)q;
    uint32_t u = 0, ph = 1;
    bool ok = true;
#pragma unroll 1
    for (int64_t t = pair; t < tiles && ok; t += pairs) {
      const Item it = tile_at(items, t);
      const int j = it.j0 + 128 * (int)rank + r;
      const uint8_t* row[3];
      bool live[3];
      live[0] = j < A.N;
      row[0] = A.ws + it.e * A.gws + (int64_t)j * A.ldws;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        live[1 + h] = 128 * h + r < it.rows;
        row[1 + h] = A.as + (it.r0 + 128 * h + r) * A.ldas;
      }
#pragma unroll 1
      for (int k = 0; k < steps; k += kUnit) {
        uint32_t v[3][2][4];
#pragma unroll
        for (int p = 0; p < 3; ++p) load_scales(v[p], row[p], live[p], whole != 0, 8 * k, len);
        ok = __all_sync(kFull, wait_phase(&sh->taken[u], ph, failed));
        if (!ok) break;
        const uint32_t to = ring + u * (uint32_t)kUnitBytes;
#pragma unroll
        for (int z = 0; z < kUnit; ++z)
#pragma unroll
          for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int p = 0; p < 3; ++p)   // channels' two cells; of either 128 codes the rows' two halves
              sts32(to + (uint32_t)(kCells * z + kCell * (p == 0 ? y : 2 + 2 * y + (p - 1))), v[p][z >> 1][2 * (z & 1) + y]);
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh->loaded[u]);
        if (++u == kUnits) {
          u = 0;
          ph ^= 1u;
        }
      }
    }
  } else if (warp < kMmaWarp) {
    // ---------------- scales to tensor memory ----------------
    // Every quarter of the lanes holds all of a cell: lane i the 16 bytes at 16 i, in four columns.
    const uint32_t ring = smem_u32(base) + (uint32_t)(kStages * kStageBytes) + 16u * (uint32_t)lane;
    const uint32_t sf0 = tmem + ((uint32_t)(32 * (warp & 3)) << 16) + (uint32_t)kSfCol;
    uint32_t u = 0, ph = 0, slot = 0, old = 0, oph = 0;   // (old: the stage kSlots steps before)
    int fresh = kSlots;                                   // slots that nothing has read yet
    bool ok = true;
#pragma unroll 1
    for (int64_t t = pair; t < tiles && ok; t += pairs) {
#pragma unroll 1
      for (int k = 0; k < steps && ok; k += kUnit) {
        ok = __all_sync(kFull, wait_phase(&sh->loaded[u], ph, failed));
        const int some = min(kUnit, steps - k);
#pragma unroll 1
        for (int z = 0; z < some && ok; ++z) {
          const uint32_t from = ring + u * (uint32_t)kUnitBytes + (uint32_t)(kCells * z);
          uint32_t f[8], g[16];
#pragma unroll
          for (int e = 0; e < 2; ++e) lds_cell(&f[4 * e], from + (uint32_t)(kCell * e));
#pragma unroll
          for (int e = 0; e < 4; ++e) lds_cell(&g[4 * e], from + (uint32_t)(kCell * (2 + e)));
          // the MMAs that read the scales in this slot
          if (fresh > 0) {
            --fresh;
          } else {
            ok = __all_sync(kFull, wait_phase<kOrder>(&sh->empty[old], oph, failed));
            if (!ok) break;
            if (++old == kStages) {
              old = 0;
              oph ^= 1u;
            }
          }
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          tmem_store8(sf0 + (uint32_t)kSlotCols * slot, f);
          tmem_store16(sf0 + (uint32_t)kSlotCols * slot + 8u, g);
          asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
          asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
          __syncwarp();
          if (lane == 0) {
            mbar_arrive_rank0(&sh->scaled[slot]);
            if (z + 1 == some) mbar_arrive(&sh->taken[u]);
          }
          if (++slot == kSlots) slot = 0;
        }
        if (++u == kUnits) {
          u = 0;
          ph ^= 1u;
        }
      }
    }
  } else if (warp == kCopyWarp) {
    // ---------------- copies ----------------
    if (lane == 0) {
      uint32_t s = 0, ph = 1;
      int64_t copied = 0;
      bool ok = true;
#pragma unroll 1
      for (int64_t t = pair; t < tiles && ok; t += pairs) {
        const Item it = tile_at(items, t);
        const int half = (it.rows + 31) / 32 * 16;   // rows of a CTA
        const int wy = it.j0 + 128 * (int)rank, ay = (int)it.r0 + half * (int)rank;
#pragma unroll 1
        for (int k = 0; k < steps; ++k) {
          ok = wait_phase<kPeer>(&sh->empty[s], ph, failed);
          if (!ok) break;
          const uint32_t to = smem_u32(base) + s * (uint32_t)kStageBytes, bar = rank0_address(&sh->full[s]);
          if (rank == 0) mbar_arrive_tx(&sh->full[s], 4 * kBlockBytes);
          copy_w(to, &maps.w, k * kStepBytes, wy, it.e, bar);
          copy_a(to + kBlockBytes, &maps.a, k * kStepBytes, ay, bar);
          ++copied;
          if (++s == kStages) {
            s = 0;
            ph ^= 1u;
          }
        }
      }
      // The last stages' MMAs: the arrivals of their commits, to both CTAs, are not under way when one leaves.  After an
      // expired wait the even CTA waits for the copies: none outlives its CTA, and the last phases hold both
      // CTAs' (where the odd one stopped earlier, the wait's limit is time enough for what is in flight).
      unsigned long long* last = ok || rank != 0 ? sh->empty : sh->full;
      volatile int late = 0;   // (of its own: the MMAs' last wait goes on after one of these expires)
      for (int64_t k = copied > kStages ? copied - kStages : 0; k < copied; ++k)
        wait_phase<kPeer>(&last[k % kStages], (uint32_t)(k / kStages) & 1u, &late, ok ? kWaitCycles : 2000000ull);
    }
  } else if (rank == 0) {
    // ---------------- MMAs of the pair ----------------
    const bool lead = elect_one();
    const uint32_t d = uniform(tmem);
    const uint64_t desc0 = smem_desc(uniform(smem_u32(base)));
    uint32_t s = 0, ph = 0, slot = 0, sph = 0, made = 0;
    bool ok = true;
#pragma unroll 1
    for (int64_t t = pair; t < tiles && ok; t += pairs, ++made) {
      const Item it = tile_at(items, t);
      const uint32_t acc = d + (made & 1u) * (uint32_t)(TP - kShared);
      const uint32_t idesc = uniform(idesc_f4(TP, (it.rows + 31) & ~31));
      // the columns that this accumulator shares with the one before are read, and all of its own
      // were before those
      if (made > 0) ok = __all_sync(kFull, wait_phase<kOrder>(&sh->drained, (made - 1) & 1u, failed));
      if (!ok) break;
#pragma unroll 1
      for (int k = 0; k < steps; ++k) {
        ok = __all_sync(kFull, wait_phase<kOrder>(&sh->scaled[slot], sph, failed));
        ok = ok && __all_sync(kFull, wait_phase<kPeer>(&sh->full[s], ph, failed));
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint64_t ad = desc0 + (uint64_t)(s * (uint32_t)(kStageBytes >> 4)), bd = ad + (uint64_t)(kBlockBytes >> 4);
        const uint32_t sf = d + (uint32_t)kSfCol + (uint32_t)kSlotCols * slot;
        const int left = (int)min((int64_t)kStepBytes, bytes - (int64_t)k * kStepBytes);
        if (lead) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (e == 0 || left > 32 * e)
              mma_mx4_pair(acc, ad + 2 * e, bd + 2 * e, idesc | (uint32_t)((e & 1) * 2) << 4 | (uint32_t)((e & 1) * 2) << 29,
                           sf + 4 * (e >> 1), sf + 8 + 8 * (e >> 1), (k > 0 || e > 0) ? 1u : 0u);
          mma_commit_pair(&sh->empty[s]);
        }
        __syncwarp();
        if (++slot == kSlots) {
          slot = 0;
          sph ^= 1u;
        }
        if (++s == kStages) {
          s = 0;
          ph ^= 1u;
        }
      }
      if (ok && lead) mma_commit_pair(&sh->done[made & 1u]);
      __syncwarp();
    }
    if (lead) {
      // no MMA outlives its operands and its tensor memory
      mma_commit_pair(&sh->left);
      wait_phase(&sh->left, 0, &sh->left_failed);
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
  if (rank != 0 && threadIdx.x == 0) wait_phase<kPeer>(&sh->left, 0, &sh->left_failed);
  __syncwarp();
  pair_sync();
  if (redo) {
    for (int64_t t = pair; t < tiles; t += pairs) {
      Item it = tile_at(items, t);
      it.j0 += 128 * (int)rank;
      plain_rows(A, it, 0, 1);
    }
  }
}

template <typename TOut>
cudaError_t launch_pair(const Mx4Args& A, const Maps& maps, cudaStream_t st, int expire) {
  static std::atomic<uint64_t> done{0};
  const cudaError_t e = allow_smem(done, k_mx4_pair<TOut>, 227 * 1024);
  if (e != cudaSuccess) return e;
  const int ctiles = (int)(((int64_t)A.N + TP - 1) / TP);
  const int64_t some = A.offsets ? std::min<int64_t>(A.E, A.n) : 1;
  const int64_t rtiles = A.offsets ? some + (A.n - some) / TP : (A.n + TP - 1) / TP;   // at most
  const int64_t pairs = std::min<int64_t>(sm_count() / 2, ctiles * rtiles);
  return launch_kernel(k_mx4_pair<TOut>, dim3((unsigned)(2 * pairs)), dim3(kThreads), (size_t)pair_smem(A.offsets ? A.E : 0), st,
                       true, A, maps, ctiles, (int)scales_whole(A), expire);
}

}  // namespace

cudaError_t launch_mx4_pair(const Mx4Args& A, const mx4::Maps& maps, cudaStream_t st, int expire) {
  static_assert(pair_smem(kPairGroups) <= 227 * 1024, "shared memory");
  if (A.type == BMLP_F32) return launch_pair<float>(A, maps, st, expire);
  if (A.type == BMLP_F16) return launch_pair<__half>(A, maps, st, expire);
  return launch_pair<__nv_bfloat16>(A, maps, st, expire);
}

}  // namespace bk
