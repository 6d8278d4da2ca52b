// kern_int8.cu -- product of 8-bit integers, S = a w^T, exact in int32, with scales
// per row and channel or as packed signs against thresholds: the choice of kernel.
#include "bmlp_internal.cuh"

#include <algorithm>

namespace bk {
namespace {

enum class Path { kFew, kTiles, kReadyTiles, kPairs };
struct Plan {
  Path path;
  int nt;      // rows of a tile
  bool swap;   // rows and channels change places
};

int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Which kernel: the least of the times that lines give each, fitted to measurements of every plan
// at 290 sizes; at 290 others the chosen plan's times are 0.8% above the best's in the mean, 27% at
// worst (some of the first below, in us).  The lines know nothing of what eight CTAs that share K gain and
// how many clusters run at once (kern_int8_tile.cu): 300 x 16384 -> 384 17.7, 32-row tiles 15.9;
// 50 x 1243 -> 2331 11.9, 64-row tiles 7.9.  Tiles: a launch and what follows the last sum; per k-step of 128 codes; per
// further round where there are more tiles than SMs; the tiles' rows made ready.  Rows at odd places:
// K not a multiple of 16 stands for them (the size of the workspace goes by the sizes alone; at 13
// sizes of whole K in rows at odd places the chosen plan was the best of all).
//                         32-row tiles  64, ready  128, ready  pairs  swapped 32, 64, 128
//   200 x 1024 -> 1024 and smaller: 32-row tiles (172 x 208 -> 224 3.6, 5.3, 6.0, 9.7)
//   46 x 4320 -> 7472             16.6       14.2           -      -
//   100 x 4096 -> 8192            30.2       18.8        15.6      -
//   300 x 12144 -> 8208            198        127          89    140
//   2478 x 1600 -> 8415            287        156          91     67
//   13230 x 1696 -> 272             92         69          49     46     62, 41, 34
//   36560 x 12548 -> 35            980        907         716    528     307, 119, -
//   16084 x 128 -> 2192 signs      205        105          67     30     221, 111, 63
// Up to 8 rows the streamed kernel: 8 x 8192 -> 8192 14.8 (32-row 17.0), 1 x 784 -> 2048 2.8 (5.3).
Plan plan_of(int64_t n, int K, int N) {
  if (n <= 8) return {Path::kFew, 0, false};
  const bool odd = K % 16 != 0;
  Plan p = {Path::kTiles, 32, false};
  double best = 1e30;
  for (int swap = 0; swap < 2; ++swap) {
    const int64_t rows = swap ? N : n, channels = swap ? n : N;
    if (swap && (n > (1 << 30) || N > kTileSlab || n <= N)) continue;
    auto tiles = [&](Path path, int nt, double start, double per_step, double per_round) {
      const int64_t t = up(channels, 128) * up(rows, nt);
      const int split = int8_tile_split(t, K, nt, swap);
      const double steps = (double)up(K, 128) / split, rounds = (double)up(t * split, sm_count());
      const double ready = path == Path::kReadyTiles ? 3.0 * (double)rows * K / 4.5e6 : 0;
      const double us = start + ready + rounds * steps * per_step + (rounds - 1) * per_round + 0.3 * swap * rounds;
      if (us < best) p = {path, nt, swap != 0}, best = us;
    };
    tiles(Path::kTiles, 32, 3.1, odd ? 1.03 : 0.46, 3.3);
    if (rows > 32) tiles(Path::kReadyTiles, 64, odd ? 5.5 : 5.1, odd ? 0.60 : 0.43, 3.9);
    if (rows > 64) tiles(Path::kReadyTiles, 128, 6.7, odd ? 0.59 : 0.42, 5.1);
  }
  // pairs; up to K = 1024 a tile's outputs go out as they are read
  const int64_t pairs = up(up(N, 256) * up(n, 256), sm_count() / 2);
  const double us = 10.8 + 3.0 * ((double)n + N) * K / 4.5e6 + (double)pairs * std::max(K <= 1024 ? 3.3 : 10.0, (double)up(K, 64) * 0.27);
  // (blocks are numbered in 31 bits)
  if (((int64_t)N + 256) * (K / 64 + 1) < (1ll << 31) && n > 128 && us < best) p = {Path::kPairs, 0, false};
  return p;
}

int64_t workspace_of(const Plan& p, int64_t n, int K, int N) {
  return p.path == Path::kReadyTiles ? int8_rows_workspace(p.swap ? N : n, K)
                                     : (p.path == Path::kPairs ? int8_pair_workspace(n, K, N) : 0);
}

}  // namespace

int64_t int8_workspace(int64_t n, int K, int N) { return workspace_of(plan_of(n, K, N), n, K, N); }

cudaError_t launch_int8(const Int8Args& A, void* workspace, int64_t workspace_bytes, cudaStream_t st, int expire) {
  const Plan p = plan_of(A.n, A.K, A.N);
  if (p.path == Path::kFew) return launch_int8_few(A, st);
  if (p.path == Path::kTiles) return launch_int8_tile(A, nullptr, st, expire, p.nt, p.swap);
  if (!workspace || workspace_bytes < workspace_of(p, A.n, A.K, A.N))
    return launch_int8_tile(A, nullptr, st, expire, (p.swap ? A.N : A.n) <= 64 ? 64 : 128, p.swap);
  return p.path == Path::kPairs ? launch_int8_pair(A, workspace, st, expire)
                                : launch_int8_tile(A, workspace, st, expire, p.nt, p.swap);
}

}  // namespace bk
