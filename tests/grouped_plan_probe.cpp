// Prints what the library's host code plans for the large products of layers over stacks of experts and 8-bit weights named on stdin
// (tests/test_experts_plans.py, tests/test_gpu_experts_split.py); links librunlora.so, runs nothing on a GPU.
#include <cstdio>
#include <cstring>

#include "../paper_2312_03415_amd/csrc/grouped.hpp"

using namespace rl;

int main() {
  char kind[16];
  long a, b, c, d, e, f;
  while (std::scanf("%15s %ld %ld %ld %ld %ld %ld", kind, &a, &b, &c, &d, &e, &f) == 7) {
    if (std::strcmp(kind, "product") == 0) {  // rows, experts, columns, K, 8-bit, ends are given: tile's rows and columns, join
      ExpertsDesc x;
      x.n = a; x.experts = b; x.f8 = e != 0; x.has_ends = f != 0;
      const GroupedPlan p = grouped_plan(x, c, d, false);
      const GroupedTileInfo t = grouped_tile(p.tile);
      std::printf("%d %d %d\n", t.bm, t.bn, p.join ? 1 : 0);
    } else if (std::strcmp(kind, "few") == 0) {  // the same product for few rows: slices of K
      ExpertsDesc x;
      x.n = a; x.experts = b; x.f8 = e != 0; x.has_ends = f != 0;
      std::printf("%d\n", grouped_plan(x, c, d, true).splits);
    } else if (std::strcmp(kind, "split") == 0) {  // 256 x 256 tiles, K tiles: tiles that stay whole, runs a tile and K tiles a run of the others
      const GroupedSplit s = grouped_split_round((int)a, (int)b);
      std::printf("%d %d %d\n", s.whole, s.splits, s.per);
    }
  }
  return 0;
}
