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

// Which kernel: the least of the times that a line through measurements gives each (us; with
// what was measured beside it).  Tiles: a launch and what follows the last sum, and per k-step of
// 128 codes; the tiles' rows made ready; more tiles than SMs run in rounds.  Rows at odd places: K not a multiple of 16 stands
// for them (the size of the workspace goes by the sizes alone).
//   32-row tiles      32 x 8192 -> 8192 16.6, 32 x 4096 -> 4096 7.8, 200 x 1024 -> 1024 6.0
//   64, ready rows    64 x 8192 -> 8192 20.1 (32-row 26.5, 128-row 22.6), 500 x 1000 -> 1000 9.0 (9.6, 9.7)
//   128, ready rows   100 x 4096 -> 8192 15.5 (31, 18.3; pairs 46), 300 x 8192 -> 8192 61 (132, 86; 88),
//                     700 x 4096 -> 4096 36 (78, 50; 38.5)
//   pairs             1500 x 1024 -> 8192 36 (128-row 46), 2000 x 4096 -> 4096 63 (73)
//   swapped           17871 x 4646 -> 78 32 (158), 33078 x 2816 -> 448 94 (154), 1000 x 1000 -> 525 11.2 (14.2);
//                     47454 x 119 -> 35 25 (20.5), the line's worst here
// Up to 8 rows the streamed kernel: 8 x 8192 -> 8192 14.8 (32-row 17.0), 1 x 784 -> 2048 2.8 (5.3).
Plan plan_of(int64_t n, int K, int N) {
  if (n <= 8) return {Path::kFew, 0, false};
  const double odd = K % 16 ? 1.0 : 0.0;
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
      const double us = start + 1.5 * odd + ready + rounds * steps * per_step * (1 + 0.3 * odd) + (rounds - 1) * per_round;
      if (us < best) p = {path, nt, swap != 0}, best = us;
    };
    tiles(Path::kTiles, 32, 4.6, 0.36, 2.5);
    if (rows > 32) tiles(Path::kReadyTiles, 64, 6.1, 0.44, 2.5);
    if (rows > 64) tiles(Path::kReadyTiles, 128, 7.4, 0.50, 1.5);
  }
  // pairs; up to K = 1024 a tile's outputs go out as they are read
  const int64_t pairs = up(up(N, 256) * up(n, 256), sm_count() / 2);
  const double tile = std::max(K <= 1024 ? 3.0 : 4.5, (double)up(K, 64) * 0.27);
  const double us = 8.0 + 3.0 * ((double)n + N) * K / 4.5e6 + 3.5 + (double)pairs * tile;
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
