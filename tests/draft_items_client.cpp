// Reads cases from its input and prints in which order a tree's items take its row tiles and splits (built and run by tests/test_draft_items.py).
#include <cstdio>

#include "attend_plan.h"

int main() {
  unsigned Hk, tiles, splits;
  while (std::scanf("%u %u %u", &Hk, &tiles, &splits) == 3) {
    for (unsigned e = 0; e < Hk * tiles * splits; ++e) {
      uint32_t tile, split;
      asl::tree_turn(e, Hk, tiles, splits, &tile, &split);
      std::printf("%u %u ", tile, split);
    }
    std::printf("\n");
  }
  return 0;
}
