// kern_mx4_tile.cu -- the product of microscaled 4-bit rows on the tensor cores,
//   y_ij = row_scale_i sum_b 2^(sa_ib + sw_jb - 254) sum_{k in block b} a_ik w_jk + bias_j,
// with one matrix of weights or that of each row's group: tiles of one CTA, and the choice of kernel.
//
// The codes lie in memory as tcgen05.mma kind::mxf4 wants them in shared memory (K-major, two
// to a byte), so tensor copies take them there, zeros past the operands' ends, and nobody
// touches them on the way.  A CTA computes 128 channels (MMA M; lanes of tensor memory) x up to
// 128 rows (MMA N, as many as the tile has, up to 16); channels on M: a narrow batch costs narrow MMAs,
// and a warp's lanes hold 32 neighbouring channels of a row, as the output wants them.
// Warps:
//   - one thread copies stages of 256 codes of every row into a ring (rows at places that
//     tensor copies cannot take: four warps copy the 16-byte chunks around them, and eight shift those to their places);
//   - eight warps, four at a time, load the scales of 1024 codes (32 bytes) of every row, a row each lane's
//     own, and store them to the stages as cells of 128 rows x 128 codes: the four bytes
//     of row r at 16 (r % 32) + 4 (r / 32), which is how the MMA wants them in the lanes and
//     columns of tensor memory;
//   - one warp copies a stage's cells there, to all four quarters of the lanes;
//   - one warp issues the MMAs, 64 codes (two blocks) each;
//   - 4, 8 or 16 warps write finished tiles while the next one's MMAs run (two accumulators).
// Where there are fewer tiles than SMs, the CTAs of a cluster share K and add their sums up
// in the order of their ranks, through distributed shared memory.
// By group: the row tiles of a group start at its first row; what a tile has of the next
// group's rows is multiplied and dropped.
// Every wait is bounded; if one expires the CTA's tiles are made again on CUDA cores.
// Measured (us): 1 x 8192 -> 8192 10.6, 100 x 4096 -> 8192 9.2, 96 x 4096 -> 2048 by 32 26, rows of 500 bytes at
// odd places 1000 x 1000 -> 525 9.2.  A step of 256 codes takes 600 clocks where its MMAs (128 rows)
// take 256: a tensor copy brings a row's 128 bytes in 2.4 clocks.
#include <algorithm>
#include <cmath>

#include <cuda.h>

#include "mx4_common.cuh"

namespace bk {
namespace {

using namespace tc;
using namespace mx4;

constexpr int CM = 128;                  // channels of a tile
constexpr int kMaxRows = 128;
constexpr int kTwoRows = 32;             // rows of a tile up to which an SM has two CTAs
constexpr int kStepBytes = 128;          // of a row per stage: 256 codes
constexpr int kScaleWarps = 4;           // of a group; two groups
constexpr int kRawWarps = 4, kShiftWarps = 8;
constexpr int kRawRow = kStepBytes + 16; // of a row at any place: the chunks around 128 bytes
constexpr int kMaxDeep = 6;              // steps of them in the ring
constexpr int kMaxStages = 8;
constexpr int kCells = 4 * kCell;        // of a stage: two of the channels, two of the rows
constexpr int kSlotCols = 16;            // of tensor memory for them
constexpr int kUnit = 4;                 // steps whose scales a lane loads at once: 32 bytes of a row

struct __align__(8) TileShared {
  unsigned long long scaled[kMaxStages], full[kMaxStages], empty[kMaxStages];   // cells; codes, and scales in tensor memory; read
  unsigned long long raw_full[kMaxDeep], raw_empty[kMaxDeep];
  unsigned long long done[2], drained[2];
  unsigned long long left, cells_left;
  uint32_t tmem_base;
  int failed, left_failed;
};

struct TilePlan {
  int nt;          // rows of a tile, a multiple of 16
  int stages;
  int deep;        // steps in the ring of rows that start anywhere; 0: tensor copies
  int cols;        // of tensor memory
  int split;       // CTAs that share K
  int ctiles;      // channel tiles
  int ctas;        // of the grid
  int whole;       // every row's scales start at a multiple of 16 bytes
};

__host__ __device__ constexpr int stage_size(int nt) { return (CM + nt) * kStepBytes + kCells; }
int64_t tile_smem(const Mx4Args& A, int nt, int stages, int deep) {
  return 1024 + (int64_t)deep * kRawRow * (CM + nt) + (int64_t)stages * stage_size(nt) + (int64_t)sizeof(TileShared) +
         (A.offsets ? 8 * ((int64_t)A.E + 1) : 0);
}

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t peer_addr(uint32_t local_addr, uint32_t rank) {
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(local_addr), "r"(rank));
  return a;
}
__device__ __forceinline__ uint32_t peer_load(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ float4 peer_load4(uint32_t a) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a) : "memory");
  return v;
}

__device__ __forceinline__ void mma_mx4(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t sfa,
                                        uint32_t sfb, uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %6, 0;\n"
      " tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n}"
      ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate));
}

// A cell to four columns of tensor memory, 32 lanes in each quarter.
__device__ __forceinline__ void copy_cell(uint32_t tmem_to, uint64_t cell) {
  asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem_to), "l"(cell) : "memory");
}
__device__ __forceinline__ void copy_w(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
      ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
__device__ __forceinline__ void copy_a(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
      ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}

// The tiles of a CTA (or of a cluster of them), one after another: row tile u, channel tile ct.
struct Cursor {
  int64_t u;
  int ct;
  __device__ __forceinline__ Cursor(const Items& I, uint32_t first) : u(first / (uint32_t)I.ctiles), ct((int)(first % (uint32_t)I.ctiles)) {}
  __device__ __forceinline__ bool live(const Items& I) const { return u < I.rtiles; }
  __device__ __forceinline__ void next(const Items& I) {
    u += I.step_u;
    ct += I.step_c;
    if (ct >= I.ctiles) {
      ct -= I.ctiles;
      ++u;
    }
  }
  __device__ __forceinline__ Item at(const Items& I) const { return I.at(u, CM * ct); }
};

// Outputs of rows rank, rank + S, .. of a tile from the S CTAs' sums ([row][channel] at `sums` of each
// one's shared memory), added in the order of their ranks: a warp takes a row, a lane four channels.
// rs: of the warp's l-th row in lane l.  Eight loads are under way at a time.
template <typename TOut, int S>
__device__ __forceinline__ void join_sums(const Mx4Args& A, const Item& it, uint32_t rank, uint32_t sums, float rs,
                                          const float (&bias)[4]) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = (int)blockDim.x >> 5;
  constexpr int kRows = 8 / S;
  uint32_t from[S];
#pragma unroll
  for (int p = 0; p < S; ++p) from[p] = peer_addr(sums + 16u * (uint32_t)lane, (uint32_t)p);
  const int j = it.j0 + 4 * lane;
  const bool vec = j + 4 <= A.N && ((A.ldo | it.j0) & 3) == 0 && (reinterpret_cast<uintptr_t>(A.out) & (4 * sizeof(TOut) - 1)) == 0;
  int l = 0;
#pragma unroll 1
  for (int x0 = (int)rank + S * warp; x0 < it.rows; x0 += kRows * S * warps) {
    float4 f[kRows][S];
#pragma unroll
    for (int y = 0; y < kRows; ++y)
#pragma unroll
      for (int p = 0; p < S; ++p)
        if (y == 0 || x0 + y * S * warps < it.rows) f[y][p] = peer_load4(from[p] + 4u * CM * (uint32_t)(x0 + y * S * warps));
#pragma unroll
    for (int y = 0; y < kRows; ++y, ++l) {
      const int x = x0 + y * S * warps;
      const float by = __shfl_sync(kFull, rs, l);
      if (x >= it.rows) break;
      float4 sum = f[y][0];
#pragma unroll
      for (int p = 1; p < S; ++p) {
        sum.x = __fadd_rn(sum.x, f[y][p].x);
        sum.y = __fadd_rn(sum.y, f[y][p].y);
        sum.z = __fadd_rn(sum.z, f[y][p].z);
        sum.w = __fadd_rn(sum.w, f[y][p].w);
      }
      union { TOut e[4]; uint2 two; uint4 four; } out;
      const float v[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) out.e[e] = output<TOut>(v[e], by, bias[e]);
      TOut* to = static_cast<TOut*>(A.out) + (it.r0 + x) * A.ldo + j;
      if (vec) {
        if constexpr (sizeof(TOut) == 4) *reinterpret_cast<uint4*>(to) = out.four;
        else *reinterpret_cast<uint2*>(to) = out.two;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (j + e < A.N) to[e] = out.e[e];
      }
    }
  }
}

// 16 bytes, past L1.
__device__ __forceinline__ void copy16(uint32_t to, const int8_t* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}

// kTma: the codes come by tensor copies (else their rows start anywhere).  kEpiWarps: that write outputs.
__device__ __forceinline__ int64_t up_steps(int K) { return (((int64_t)K + 1) / 2 + kStepBytes - 1) / kStepBytes; }
template <int kEpiWarps, bool kTma> struct Warps {
  static constexpr int kMma = kEpiWarps + 2 * kScaleWarps, kCopy = kMma + 2, kAll = kCopy + (kTma ? 1 : kRawWarps + kShiftWarps);
};
template <typename TOut, int kEpiWarps, bool kTma>
__global__ void __launch_bounds__(32 * Warps<kEpiWarps, kTma>::kAll, kTma && kEpiWarps == 4 ? 2 : 1)
    k_mx4_tile(const Mx4Args A, const __grid_constant__ Maps maps, const TilePlan P, int expire) {
  constexpr int kMmaWarp = Warps<kEpiWarps, kTma>::kMma, kCellWarp = kMmaWarp + 1, kCopyWarp = kCellWarp + 1;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  const int stage_bytes = stage_size(P.nt);
  uint8_t* ring = base + P.stages * stage_bytes;
  TileShared* sh = reinterpret_cast<TileShared*>(ring + P.deep * kRawRow * (CM + P.nt));
  int32_t* groups = reinterpret_cast<int32_t*>(sh + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t S = (uint32_t)P.split, rank = S > 1 ? cluster_rank() : 0u;
  volatile int* failed = &sh->failed;

  if (threadIdx.x == 0) {
    for (int s = 0; s < P.stages; ++s) {
      mbar_init(&sh->full[s], 1 + (kTma ? 1 : kShiftWarps));
      mbar_init(&sh->scaled[s], kScaleWarps);
      mbar_init(&sh->empty[s], 1);
    }
    for (int s = 0; s < P.deep; ++s) {
      mbar_init(&sh->raw_full[s], 32 * kRawWarps);
      mbar_init(&sh->raw_empty[s], kShiftWarps);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&sh->done[b], 1);
      mbar_init(&sh->drained[b], kEpiWarps);
    }
    mbar_init(&sh->left, 1);
    mbar_init(&sh->cells_left, 1);
    sh->failed = sh->left_failed = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                 ::"r"(smem_u32(&sh->tmem_base)), "r"(P.cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (kTma && warp == kCopyWarp && lane == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.w) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.a) : "memory");
    // the first stages' weights on their way to L2 while the launch before this one ends
    if (!A.offsets) {
      const int ks = (int)up_steps(A.K), chunks0 = (ks + 1) / 2, from = 2 * (int)((int64_t)chunks0 * rank / S);
      const int to = min(min(2 * (int)((int64_t)chunks0 * (rank + 1) / S), ks), from + P.stages);
      const int j0 = CM * (int)((blockIdx.x / S) % (uint32_t)P.ctiles);
      for (int k = from; k < to; ++k)
        asm volatile("cp.async.bulk.prefetch.tensor.3d.L2.global.tile [%0, {%1, %2, %3}];"
                     ::"l"(&maps.w), "r"(k * kStepBytes), "r"(j0), "r"(0) : "memory");
    }
  }
  pdl_wait();
  pdl_trigger();
  if (A.offsets && warp == 0) group_tiles(A, P.nt, groups);
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = sh->tmem_base;
  const uint32_t first = blockIdx.x / S, step = gridDim.x / S;
  const Items items = {A.offsets ? groups : nullptr, A.offsets ? groups + A.E + 1 : nullptr, A.E, P.nt, P.ctiles,
                       (int)(step / (uint32_t)P.ctiles), (int)(step % (uint32_t)P.ctiles),
                       A.offsets ? (int64_t)groups[A.E] : (A.n + P.nt - 1) / P.nt, A.n};
  // this CTA's k-steps [k0, k1): whole chunks of two
  const int64_t bytes = ((int64_t)A.K + 1) / 2;
  const int steps = (int)((bytes + kStepBytes - 1) / kStepBytes), chunks = (steps + 1) / 2;
  const int c0 = (int)((int64_t)chunks * rank / S), c1 = (int)((int64_t)chunks * (rank + 1) / S);
  const int k0 = 2 * c0, k1 = min(2 * c1, steps);

  if (warp < kEpiWarps) {
    // ---------------- outputs ----------------
    constexpr int kParts = kEpiWarps / 4, kEach = (kTma && kEpiWarps == 4 ? kTwoRows : kMaxRows) / 16 / kParts;   // blocks of 16 rows: part, part + kParts, ..
    const int quarter = warp & 3, part = warp >> 2;
    const bool has_rs = A.row_scale != nullptr, has_bias = A.bias != nullptr;
    bool ok = true;
    uint32_t seen = 0;
#pragma unroll 1
    for (Cursor at(items, first); at.live(items) && ok; at.next(items), ++seen) {
      const Item it = at.at(items);
      const int j = it.j0 + 32 * quarter + lane;
      const bool live = j < A.N;
      // what the outputs need from memory, asked for before the sums are there
      const float bias = has_bias && live ? A.bias[it.e * A.ldb + j] : 0.0f;
      float rs[kEach];
#pragma unroll
      for (int c = 0; c < kEach; ++c) {
        const int x = 16 * (kParts * c + part) + (lane & 15);
        rs[c] = has_rs && x < it.rows ? A.row_scale[it.r0 + x] : 1.0f;
      }
      const uint32_t b = seen & 1u, tacc = tmem + ((uint32_t)(32 * quarter) << 16) + b * (uint32_t)P.nt;
      ok = __all_sync(kFull, wait_phase(&sh->done[b], (seen >> 1) & 1u, failed));
      if (!ok) break;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
      for (int c = 0; c < kEach; ++c) {
        const int x0 = 16 * (kParts * c + part);
        if (x0 >= it.rows) break;
        uint32_t v[16];
        tmem_load16(v, tacc + (uint32_t)x0);
        tmem_wait_ld(v);
        if (S > 1) {
          float* to = reinterpret_cast<float*>(base) + x0 * CM + 32 * quarter + lane;
#pragma unroll
          for (int x = 0; x < 16; ++x) to[x * CM] = __uint_as_float(v[x]);
        } else if (!expire) {
          put_rows(static_cast<TOut*>(A.out) + (it.r0 + x0) * A.ldo + j, A.ldo, v, rs[c], bias, it.rows - x0, live);
        }
      }
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh->drained[b]);
    }
    if (expire && threadIdx.x == 0) *failed = 1;
  } else if (warp < kMmaWarp) {
    // ---------------- scales ----------------
    // Two groups of warps take units of 1024 codes in turn: the one loads while the other waits for
    // stages and fills them.
    const int q = (warp - kEpiWarps) & (kScaleWarps - 1), r = 32 * q + lane;   // this lane's channel and row
    const bool second = warp >= kEpiWarps + kScaleWarps, has_row = r < P.nt, whole = P.whole != 0;
    const int len = (int)(((int64_t)A.K + 31) / 32);
    const uint32_t cells = smem_u32(base) + (uint32_t)(stage_bytes - kCells) + 16u * (uint32_t)lane + 4u * (uint32_t)q;
    // A wait knows a phase by its parity alone, so the phase two before it must be known to be over.  A unit's
    // first step waits for the MMAs of P.stages steps before, hence those of 2 P.stages before must be done;
    // this group's last wait tells that of those of kUnit + 1 + P.stages before.  Shorter rings have one group.
    const bool alone = P.stages <= kUnit;
    Place at = {0, 1u};
    bool ok = true, mine = !second;
#pragma unroll 1
    for (Cursor cur(items, first); cur.live(items) && ok; cur.next(items)) {
      const uint8_t *wrow = nullptr, *arow = nullptr;
      bool wlive = false, alive = false, known = false;
#pragma unroll 1
      for (int k = k0; k < k1 && ok; k += kUnit, mine = mine == alone) {
        if (!mine) {
          at.forward(min(kUnit, k1 - k), P.stages);
          continue;
        }
        if (!known) {
          const Item it = cur.at(items);
          wlive = it.j0 + r < A.N;
          alive = r < it.rows;
          wrow = A.ws + it.e * A.gws + (int64_t)(it.j0 + r) * A.ldws;
          arow = A.as + (it.r0 + r) * A.ldas;
          known = true;
        }
        uint32_t w[2][4], a[2][4];
        load_scales(w, wrow, wlive, whole, 8 * k, len);
        load_scales(a, arow, alive, whole, 8 * k, len);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if (!ok || k + 2 * h >= k1) break;
          // two stages at a time where the ring is long: the fence takes 200 clocks
          const bool two = k + 2 * h + 1 < k1, both = two && !alone;
          const Place p0 = at;
          at.forward(1, P.stages);
          const Place p1 = at;
          if (two) at.forward(1, P.stages);
          auto put = [&](int s, int y0) {
            const uint32_t to = cells + (uint32_t)(s * stage_bytes);
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              sts32(to + (uint32_t)(kCell * y), w[h][y0 + y]);
              if (has_row) sts32(to + (uint32_t)(kCell * (2 + y)), a[h][y0 + y]);
            }
          };
          ok = __all_sync(kFull, wait_phase(&sh->empty[p0.s], p0.ph, failed));
          if (both) ok = ok && __all_sync(kFull, wait_phase(&sh->empty[p1.s], p1.ph, failed));
          if (!ok) break;
          put(p0.s, 0);
          if (both) put(p1.s, 2);
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(&sh->scaled[p0.s]);
            if (both) mbar_arrive(&sh->scaled[p1.s]);
          }
          if (two && !both) {
            ok = __all_sync(kFull, wait_phase(&sh->empty[p1.s], p1.ph, failed));
            if (!ok) break;
            put(p1.s, 2);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh->scaled[p1.s]);
          }
        }
      }
    }
  } else if (warp == kMmaWarp) {
    // ---------------- MMAs ----------------
    const bool lead = elect_one();
    const uint32_t d = uniform(tmem);
    const uint64_t desc0 = smem_desc(uniform(smem_u32(base)));
    const uint32_t sf0 = d + 2u * (uint32_t)P.nt;
    uint32_t s = 0, ph = 0, made = 0;
    bool ok = true;
#pragma unroll 1
    for (Cursor at(items, first); at.live(items) && ok; at.next(items), ++made) {
      const Item it = at.at(items);
      const uint32_t b = made & 1u, acc = d + b * (uint32_t)P.nt;
      const uint32_t idesc = uniform(idesc_f4(CM, (it.rows + 15) & ~15));
      ok = __all_sync(kFull, wait_phase(&sh->drained[b], ((made >> 1) & 1u) ^ 1u, failed));
      if (!ok) break;
#pragma unroll 1
      for (int k = k0; k < k1; ++k) {
        ok = __all_sync(kFull, wait_phase(&sh->full[s], ph, failed));
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint64_t ad = desc0 + (uint64_t)(s * (uint32_t)(stage_bytes >> 4)), bd = ad + (uint64_t)(CM * kStepBytes >> 4);
        const uint32_t sf = sf0 + (uint32_t)kSlotCols * s;
        const int left = (int)min((int64_t)kStepBytes, bytes - (int64_t)k * kStepBytes);
        if (lead) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (e == 0 || left > 32 * e)
              mma_mx4(acc, ad + 2 * e, bd + 2 * e, idesc | (uint32_t)((e & 1) * 2) << 4 | (uint32_t)((e & 1) * 2) << 29,
                      sf + 4 * (e >> 1), sf + 8 + 4 * (e >> 1), (k > k0 || e > 0) ? 1u : 0u);
          mma_commit(&sh->empty[s]);
        }
        __syncwarp();
        if (++s == (uint32_t)P.stages) {
          s = 0;
          ph ^= 1u;
        }
      }
      if (ok && lead) mma_commit(&sh->done[b]);
      __syncwarp();
    }
    if (lead) {
      // no MMA outlives its operands and its tensor memory
      mma_commit(&sh->left);
      wait_phase(&sh->left, 0, &sh->left_failed);
    }
    __syncwarp();
  } else if (warp == kCellWarp) {
    // ---------------- scales to tensor memory ----------------
    // (by the MMA warp a step took 700 clocks of its issue, 53 a copy or MMA)
    const bool lead = elect_one();
    const uint64_t cells0 = cell_desc(uniform(smem_u32(base) + (uint32_t)(stage_bytes - kCells)));
    const uint32_t sf0 = uniform(tmem) + 2u * (uint32_t)P.nt;
    uint32_t s = 0, ph = 0;
    bool ok = true;
#pragma unroll 1
    for (Cursor at(items, first); at.live(items) && ok; at.next(items)) {
#pragma unroll 1
      for (int k = k0; k < k1; ++k) {
        ok = __all_sync(kFull, wait_phase(&sh->scaled[s], ph, failed));
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        if (lead) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            copy_cell(sf0 + (uint32_t)kSlotCols * s + 4 * e, cells0 + (uint64_t)(s * (uint32_t)(stage_bytes >> 4) + e * (kCell >> 4)));
          mma_commit(&sh->full[s]);
        }
        __syncwarp();
        if (++s == (uint32_t)P.stages) {
          s = 0;
          ph ^= 1u;
        }
      }
    }
    if (lead) {
      mma_commit(&sh->cells_left);
      wait_phase(&sh->cells_left, 0, &sh->left_failed);
    }
    __syncwarp();
  } else if constexpr (kTma) {
    // ---------------- copies ----------------
    if (lane == 0) {
      uint32_t s = 0, ph = 1;
      int64_t copied = 0;
      bool ok = true;
#pragma unroll 1
      for (Cursor at(items, first); at.live(items) && ok; at.next(items)) {
        const Item it = at.at(items);
#pragma unroll 1
        for (int k = k0; k < k1; ++k) {
          ok = wait_phase(&sh->empty[s], ph, failed);
          if (!ok) break;
          const uint32_t to = smem_u32(base + s * stage_bytes), bar = smem_u32(&sh->full[s]);
          mbar_arrive_tx(&sh->full[s], (uint32_t)(stage_bytes - kCells));
          copy_w(to, &maps.w, k * kStepBytes, it.j0, it.e, bar);
          copy_a(to + CM * kStepBytes, &maps.a, k * kStepBytes, (int)it.r0, bar);
          ++copied;
          if (++s == (uint32_t)P.stages) {
            s = 0;
            ph ^= 1u;
          }
        }
      }
      if (!ok) {
        // no copy outlives its CTA (a phase may lack the scales' arrival, and then the wait's limit is
        // time enough; the flag is of its own: the MMAs' and cells' last waits go on after that)
        volatile int late = 0;
        for (int64_t k = copied > P.stages ? copied - P.stages : 0; k < copied; ++k)
          wait_phase(&sh->full[k % P.stages], (uint32_t)(k / P.stages) & 1u, &late, 2000000ull);
      }
    }
  } else {
    // ---------------- rows that start anywhere ----------------
    const int len = (int)bytes;
    const uint32_t raw0 = smem_u32(ring), raw_bytes = (uint32_t)(kRawRow * (CM + P.nt));
    uint32_t slot = 0, rph = 0;
    bool ok = true;
    if (warp < kCopyWarp + kRawWarps) {
      // Four warps copy the aligned 16-byte chunks around 128 bytes of every row to a ring.  (Not the warps that
      // fill the stages: their fence would wait for the copies ahead, a memory latency each step.)
      const int l = (int)threadIdx.x - 32 * kCopyWarp, c = l & 7, sub = l >> 3;
      const int8_t* any = i8::aligned16(reinterpret_cast<const int8_t*>(A.a));
#pragma unroll 1
      for (Cursor cur(items, first); cur.live(items) && ok; cur.next(items)) {
        const Item it = cur.at(items);
        const int8_t* w0 = reinterpret_cast<const int8_t*>(A.w) + it.e * A.gw + (int64_t)it.j0 * A.ldw;
        const int8_t* a0 = reinterpret_cast<const int8_t*>(A.a) + it.r0 * A.lda;
        const int wlive = A.N - it.j0;
#pragma unroll 1
        for (int k = k0; k < k1; ++k) {
          ok = __all_sync(kFull, wait_phase(&sh->raw_empty[slot], rph ^ 1u, failed));
          if (!ok) break;
          const uint32_t to = raw0 + slot * raw_bytes;
          const int byte = k * kStepBytes;
          const bool inside = byte + kStepBytes + 16 <= len;   // every chunk is whole
          // (rows past the last keep whatever is there: their outputs are dropped, and no code is a NaN)
          auto part = [&](const int8_t* rows, int64_t ld, int live, uint32_t dst) {
            const int8_t* row = rows + sub * ld + byte + 16 * c;
            const uint32_t to0 = dst + (uint32_t)(kRawRow * sub + 16 * c);
            const int64_t step = 4 * kRawWarps * ld;
            if (inside) {
              int r = sub;
#pragma unroll 1
              for (; r + 12 * kRawWarps < live; r += 16 * kRawWarps) {
#pragma unroll
                for (int u = 0; u < 4; ++u, row += step) copy16(to0 + (uint32_t)(kRawRow * (r - sub + 4 * kRawWarps * u)), i8::aligned16(row));
              }
#pragma unroll 1
              for (; r < live; r += 4 * kRawWarps, row += step) copy16(to0 + (uint32_t)(kRawRow * (r - sub)), i8::aligned16(row));
            } else {
              row -= byte + 16 * c;
#pragma unroll 1
              for (int r = sub; r < live; r += 4 * kRawWarps, row += step)
                i8::copy_chunk(to0 + (uint32_t)(kRawRow * (r - sub)), row, i8::row_shift<1>(row), byte + 16 * c, len, any);
            }
            if (l < live) {
              row = rows + l * ld;
              i8::copy_chunk(dst + (uint32_t)(kRawRow * l + 128), row, i8::row_shift<1>(row), byte + 128, len, any);
            }
          };
          part(w0, A.ldw, min(CM, wlive), to);
          part(a0, A.lda, it.rows, to + (uint32_t)(kRawRow * CM));
          cp_async_arrive(&sh->raw_full[slot]);
          if (++slot == (uint32_t)P.deep) {
            slot = 0;
            rph ^= 1u;
          }
        }
      }
      cp_async_wait_all();
    } else {
      // Eight warps shift them to their places in the stages: 16 channels and nt / 8 rows each.
      const int w = warp - kCopyWarp - kRawWarps, c = lane & 7, sub = lane >> 3, mine = P.nt / kShiftWarps;
      uint32_t s = 0, ph = 1;
#pragma unroll 1
      for (Cursor cur(items, first); cur.live(items) && ok; cur.next(items)) {
        const Item it = cur.at(items);
        const int8_t* w0 = reinterpret_cast<const int8_t*>(A.w) + it.e * A.gw + (int64_t)(it.j0 + 16 * w + sub) * A.ldw;
        const int8_t* a0 = reinterpret_cast<const int8_t*>(A.a) + (it.r0 + mine * w + sub) * A.lda;
#pragma unroll 1
        for (int k = k0; k < k1; ++k) {
          ok = __all_sync(kFull, wait_phase(&sh->raw_full[slot], rph, failed));
          ok = ok && __all_sync(kFull, wait_phase(&sh->empty[s], ph, failed));
          if (!ok) break;
          const uint32_t to = smem_u32(base + s * stage_bytes), src = raw0 + slot * raw_bytes;
          auto part = [&](const int8_t* row, int64_t ld, int all, int r0) {
#pragma unroll 4
            for (int r = sub; r < all; r += 4, row += 4 * ld) {
              uint32_t lo[4], hi[4], v[4];
              i8::lds_chunk(lo, src + (uint32_t)(kRawRow * (r0 + r) + 16 * c));
              i8::lds_chunk(hi, src + (uint32_t)(kRawRow * (r0 + r) + 16 * c + 16));
              i8::merge16(v, lo, hi, i8::row_shift<1>(row));
              sts128(to + 128u * (uint32_t)(r0 + r) + 16u * (uint32_t)(c ^ ((r0 + r) & 7)), v);
            }
          };
          part(w0, A.ldw, 16, 16 * w);
          part(a0, A.lda, mine, CM + mine * w);
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(&sh->raw_empty[slot]);
            mbar_arrive(&sh->full[s]);
          }
          if (++slot == (uint32_t)P.deep) {
            slot = 0;
            rph ^= 1u;
          }
          if (++s == (uint32_t)P.stages) {
            s = 0;
            ph ^= 1u;
          }
        }
      }
    }
  }
  __syncwarp();
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  if (warp == kMmaWarp)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(P.cols) : "memory");
  if (S > 1) {
    const Cursor at(items, first);   // (one tile)
    const bool some = at.live(items);
    const Item it = some ? at.at(items) : Item{};
    const int warps = (int)blockDim.x >> 5;
    // this rank's rows are rank, rank + S, ..; lane l keeps the factor of the warp's l-th
    const int own = (int)rank + (int)S * (warp + warps * lane);
    const float rs = A.row_scale && own < it.rows ? A.row_scale[it.r0 + own] : 1.0f;
    const int j = it.j0 + 4 * lane;
    float bias[4];
#pragma unroll
    for (int y = 0; y < 4; ++y) bias[y] = A.bias && some && j + y < A.N ? A.bias[it.e * A.ldb + j + y] : 0.0f;
    cluster_sync();   // every CTA's sums are in its shared memory
    bool redo = false;
    for (uint32_t p = 0; p < S; ++p) redo |= peer_load(peer_addr(smem_u32(&sh->failed), p)) != 0u;
    if (redo) {
      if (some) plain_rows(A, it, (int)rank, (int)S);
    } else if (S == 2) {
      join_sums<TOut, 2>(A, it, rank, smem_u32(base), rs, bias);
    } else if (S == 4) {
      join_sums<TOut, 4>(A, it, rank, smem_u32(base), rs, bias);
    } else {
      join_sums<TOut, 8>(A, it, rank, smem_u32(base), rs, bias);
    }
    cluster_sync();   // no CTA leaves while its sums are read
  } else if (*failed) {
    for (Cursor at(items, first); at.live(items); at.next(items)) plain_rows(A, at.at(items), 0, 1);
  }
}

template <typename TOut, int kEpiWarps, bool kTma>
cudaError_t launch_mode(const Mx4Args& A, const TilePlan& P, const Maps& maps, cudaStream_t st, int expire) {
  static std::atomic<uint64_t> done{0};
  const cudaError_t e = allow_smem(done, k_mx4_tile<TOut, kEpiWarps, kTma>, 227 * 1024);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)P.ctas);
  cfg.blockDim = dim3(32 * Warps<kEpiWarps, kTma>::kAll);
  cfg.dynamicSmemBytes = (size_t)tile_smem(A, P.nt, P.stages, P.deep);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)P.split;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = P.split > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, k_mx4_tile<TOut, kEpiWarps, kTma>, A, maps, P, expire);
}

template <typename TOut>
cudaError_t launch_tile(const Mx4Args& A, const TilePlan& P, const Maps& maps, bool tma, cudaStream_t st, int expire) {
  if (!tma) return launch_mode<TOut, 8, false>(A, P, maps, st, expire);
  return P.nt > kTwoRows ? launch_mode<TOut, 16, true>(A, P, maps, st, expire) : launch_mode<TOut, 4, true>(A, P, maps, st, expire);
}

// What a call costs, in us, by lines fitted to measurements of every plan at some 40 sizes: a launch and
// what follows the last sum; per round of tiles its steps of 256 codes and its outputs; CTAs that share K.
// At 80 other sizes what is taken is 1.1% above the best of all plans in the mean, 13% at worst (469 x 4877 -> 2746 by
// 16 groups 29.9, by tiles of 48 rows 26.5; 1518 x 9285 -> 2772 by 4 tiles 49.7, pairs 44.1).  Far from the line:
// 1450 x 8996 -> 9399 tiles 78, pairs 53; 466 x 886 -> 1149 6.6, 9.2.
int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }
int64_t some_groups(const Mx4Args& A) { return A.offsets ? std::min<int64_t>(A.E, A.n) : 1; }
// Row tiles at most, and on average (of a group's rows the last one is half full).
int64_t most_row_tiles(const Mx4Args& A, int nt) {
  const int64_t some = some_groups(A);
  return A.offsets ? some + (A.n - some) / nt : up(A.n, nt);
}
double row_tiles(const Mx4Args& A, int nt) {
  const double some = (double)some_groups(A);
  return A.offsets ? std::max(some, (double)A.n / nt + 0.5 * some) : (double)up(A.n, nt);
}
double tile_cost(const Mx4Args& A, int nt, int split, bool tma) {
  const double ctiles = (double)up(A.N, CM), steps = (double)up(up(A.K, 256), split), sms = (double)sm_count();
  const bool two = tma && nt <= kTwoRows;
  // (clusters of eight: more than a dozen find no room at once)
  const double room = split == 8 ? 100.0 : (two ? 2 : 1) * sms;
  if (split > 1 && ((double)most_row_tiles(A, nt) * ctiles * split > room || 512ll * split > A.K)) return 1e30;
  const double ctas = row_tiles(A, nt) * ctiles * split, rounds = std::ceil(ctas / ((two ? 2 : 1) * sms));
  const double step = tma ? (two && ctas > sms ? 0.36 : 0.20 + 0.0006 * nt) : 0.88 + 0.003 * nt;
  return 4.2 + rounds * (steps * step + 0.3 + 0.008 * nt) + (split > 1 ? 2.1 + 0.05 * split : 0.0);
}
double pair_cost(const Mx4Args& A) {
  const double tiles = row_tiles(A, 256) * (double)up(A.N, 256), steps = (double)up(A.K, 256);
  return 9.0 + std::ceil(tiles / (sm_count() / 2)) * std::max(3.5, 0.4 * steps);
}

// The plan of the tiles, and whether pairs are taken in their place.
TilePlan plan_of(const Mx4Args& A, bool tma, bool& pairs) {
  TilePlan P = {};
  double best = 1e30;
  const int64_t mean = up(A.n, some_groups(A));
  for (int nt = 16; nt <= kMaxRows; nt += nt < 64 ? 16 : 32) {
    for (int split = 1; split <= 8; split *= 2) {
      const double us = tile_cost(A, nt, split, tma);
      if (us < best) {
        best = us;
        P.nt = nt;
        P.split = split;
      }
    }
    if (nt >= mean && !A.offsets) break;
  }
  pairs = tma && A.E <= kPairGroups && pair_cost(A) < best;
  P.ctiles = (int)up(A.N, CM);
  const int64_t tiles = most_row_tiles(A, P.nt) * P.ctiles;
  P.whole = scales_whole(A);
  // two CTAs of an SM where their tensor memory and registers have room
  const bool two = tma && P.nt <= kTwoRows;
  P.cols = two ? 256 : 512;
  // (the ring takes up to half)
  const int64_t all = (two ? 113 : 227) * 1024 - tile_smem(A, P.nt, 0, 0), row = kRawRow * (int64_t)(CM + P.nt);
  P.deep = tma ? 0 : (int)std::min<int64_t>(kMaxDeep, all / 2 / row);
  P.stages = (int)std::min<int64_t>(kMaxStages, (all - P.deep * row) / stage_size(P.nt));
  const int64_t slots = (two ? 2 : 1) * (int64_t)sm_count();
  P.ctas = (int)(P.split > 1 ? tiles * P.split : std::min(tiles, slots));
  return P;
}

}  // namespace

cudaError_t launch_mx4(const Mx4Args& A, cudaStream_t st, int expire, bool only_pairs) {
  const int64_t bytes = ((int64_t)A.K + 1) / 2;
  Maps maps;
  bool tma = codes_whole(A), pairs = false;
  TilePlan P = plan_of(A, tma, pairs);
  if (only_pairs) pairs = tma && A.E <= kPairGroups;
  if (tma && (!code_map(&maps.w, A.w, bytes, A.N, A.ldw, A.E, A.gw, CM) ||
              !code_map(&maps.a, A.a, bytes, A.n, A.lda, 0, 0, pairs ? 128 : P.nt))) {
    // strides that the driver gives no map for: as rows at any place
    tma = false;
    P = plan_of(A, tma, pairs);
  }
  if (only_pairs && !pairs) return cudaErrorNotSupported;
  if (pairs) return launch_mx4_pair(A, maps, st, expire);
  if (A.type == BMLP_F32) return launch_tile<float>(A, P, maps, tma, st, expire);
  if (A.type == BMLP_F16) return launch_tile<__half>(A, P, maps, tma, st, expire);
  return launch_tile<__nv_bfloat16>(A, P, maps, tma, st, expire);
}

}  // namespace bk
