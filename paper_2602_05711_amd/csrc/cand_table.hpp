// Candidate cells of the Cartesian merge for K <= 64 (select.hip, few.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace omnimoe {

// The candidate cells (a, b) with (a + 1)(b + 1) <= K for every K <= 64, row rank major, one
// list per K (the lists for K = 1 .. 64 hold 8104 cells): a constant table, so that no
// workgroup builds its list before the first row. With fewer than K rows (columns) in the grid,
// the cells with a >= Kr (b >= Kc) are skipped where the list is read.
constexpr int kCandK = 64;
constexpr int kCandCells = 8104;
struct CandTable {
  uint16_t cell[kCandCells];  // (a << 8) | b
  uint16_t first[kCandK + 2];  // list of K: cell[first[K] .. first[K + 1])
};
constexpr CandTable make_cand_table() {
  CandTable t{};
  int c = 0;
  t.first[0] = 0;
  for (int K = 1; K <= kCandK; ++K) {
    t.first[K] = (uint16_t)c;
    for (int a = 0; a < K; ++a)
      for (int b = 0; (a + 1) * (b + 1) <= K; ++b) t.cell[c++] = (uint16_t)((a << 8) | b);
  }
  t.first[kCandK + 1] = (uint16_t)c;
  return t;
}
static_assert(make_cand_table().first[kCandK + 1] == kCandCells, "candidate table size");
static __constant__ CandTable kCand = make_cand_table();

}  // namespace omnimoe
