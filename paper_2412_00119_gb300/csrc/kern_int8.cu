// kern_int8.cu -- product of 8-bit integers, S = a w^T, exact in int32, with scales
// per row and channel or as packed signs against thresholds: the choice of kernel.
#include "bmlp_internal.cuh"

#include <algorithm>

namespace bk {
namespace {

enum class Path { kFew, kTiles, kReadyTiles, kPairs };
struct Plan {
  Path path;
  int nt;   // rows of a tile
};

int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Which kernel: the least of the times that a line through measurements gives each (us; with
// what was measured beside it).  Tiles: a launch and what follows the last sum, and per k-step of
// 128 codes; more tiles than SMs run in rounds.  Rows at odd places: K not a multiple of 16 stands
// for them (the size of the workspace goes by the sizes alone).
//   32-row tiles      32 x 8192 -> 8192 16.6, 32 x 4096 -> 4096 7.8, 200 x 1024 -> 1024 6.0
//   64, ready rows    64 x 8192 -> 8192 20.1 (32-row 26.5, 128-row 22.6), 500 x 1000 -> 1000 9.0 (9.6, 9.7)
//   128, ready rows   100 x 4096 -> 8192 15.5 (31, 18.3; pairs 46), 300 x 8192 -> 8192 61 (132, 86; 88),
//                     700 x 4096 -> 4096 36 (78, 50; 38.5)
//   pairs             1500 x 1024 -> 8192 36 (128-row 46), 2000 x 4096 -> 4096 63 (73)
// Up to 8 rows the streamed kernel: 8 x 8192 -> 8192 14.8 (32-row 17.0), 1 x 784 -> 2048 2.8 (5.3).
Plan plan_of(int64_t n, int K, int N) {
  if (n <= 8) return {Path::kFew, 0};
  const double odd = K % 16 ? 1.0 : 0.0;
  const double codes = ((double)n + N) * K;
  auto tiles = [&](int nt, double start, double per_step, double per_round) {
    const int64_t t = up(N, 128) * up(n, nt);
    const int split = int8_tile_split(t, K);
    const double steps = (double)up(K, 128) / split, rounds = (double)up(t * split, sm_count());
    return start + 1.5 * odd + rounds * steps * per_step * (1 + 0.3 * odd) + (rounds - 1) * per_round;
  };
  const double t32 = tiles(32, 4.6, 0.36, 2.5), t64 = tiles(64, 6.1, 0.44, 2.5), t128 = tiles(128, 7.4, 0.50, 1.5);
  const int64_t pairs = up(up(N, 256) * up(n, 256), sm_count() / 2);
  const double tpair = 8.0 + 3.0 * codes / 4.5e6 + 3.5 + (double)pairs * std::max(K <= 1024 ? 3.0 : 4.5, (double)up(K, 64) * 0.27);
  // (blocks are numbered in 31 bits)
  const bool blocks = ((int64_t)N + 256) * (K / 64 + 1) < (1ll << 31);
  Plan p = {Path::kTiles, 32};
  double best = t32;
  if (n > 32 && t64 < best) p = {Path::kReadyTiles, 64}, best = t64;
  if (n > 64 && t128 < best) p = {Path::kReadyTiles, 128}, best = t128;
  if (blocks && n > 128 && tpair < best) p = {Path::kPairs, 0};
  return p;
}

int64_t workspace_of(const Plan& p, int64_t n, int K, int N) {
  return p.path == Path::kReadyTiles ? int8_rows_workspace(n, K) : (p.path == Path::kPairs ? int8_pair_workspace(n, K, N) : 0);
}

}  // namespace

int64_t int8_workspace(int64_t n, int K, int N) { return workspace_of(plan_of(n, K, N), n, K, N); }

cudaError_t launch_int8(const Int8Args& A, void* workspace, int64_t workspace_bytes, cudaStream_t st, int expire) {
  const Plan p = plan_of(A.n, A.K, A.N);
  if (p.path == Path::kFew) return launch_int8_few(A, st);
  if (p.path == Path::kTiles) return launch_int8_tile(A, nullptr, st, expire, p.nt);
  if (!workspace || workspace_bytes < workspace_of(p, A.n, A.K, A.N))
    return launch_int8_tile(A, nullptr, st, expire, A.n <= 64 ? 64 : 128);   // (no other width is ever better here)
  return p.path == Path::kPairs ? launch_int8_pair(A, workspace, st, expire) : launch_int8_tile(A, workspace, st, expire, p.nt);
}

}  // namespace bk
