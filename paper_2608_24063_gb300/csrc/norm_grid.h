// How the norm's gradient shares its blocks out (norm_rope.cu): host arithmetic alone.
// tests/test_norm_grid.py compiles this file.
#pragma once

#include <stdint.h>

namespace vc {

constexpr int kNormGradBlocks = 304;   // blocks of the gradient at most, two for each of 152 SMs; rows of its workspace
constexpr int kGradRows = 16;          // rows of a group, a block's turn
struct NormGradGrid {
  int nq, nk;                          // blocks of query and of key heads: nq + nk <= kNormGradBlocks
};

// Blocks of query and of key heads: by what a group of rows costs, its heads in turns of 32
// and kGroupTurns more for its angles and its first loads; no more than there are groups.
// 12544 rows of 28 + 4 heads of 128, us (cold): by the heads alone 120, so 89.
constexpr int kGroupTurns = 3;
inline NormGradGrid norm_grad_grid(int64_t n_rows, int32_t Hq, int32_t Hkv) {
  const int64_t groups = (n_rows + kGradRows - 1) / kGradRows;
  auto cost = [](int64_t H) { return H > 0 ? (H * kGradRows + 31) / 32 + kGroupTurns : (int64_t)0; };
  const int64_t cq = cost(Hq), ck = cost(Hkv);
  const int64_t most = kNormGradBlocks - (Hq > 0 ? 1 : 0);      // (one is left for the query heads)
  int64_t nk = (kNormGradBlocks * ck + cq + ck - 1) / (cq + ck);
  if (nk > most) nk = most;
  const int64_t nq = Hq > 0 ? kNormGradBlocks - nk : 0;
  NormGradGrid g;
  g.nq = (int)(nq < groups ? nq : groups);
  g.nk = (int)(nk < groups ? nk : groups);
  return g;
}

}  // namespace vc
