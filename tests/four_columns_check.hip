// Host replay of small_loss_kernel's stores of logits, w [M, V] (tile_index.h, four_columns): every column of every shard is written by one lane.  Run by tests/test_four_columns.py.
#include <cstdio>
#include <vector>

#include "../paper_2105_04663_amd/csrc/tile_index.h"

using namespace gspmd;

int main() {
  for (int per = 8; per <= 1280; ++per) {
    std::vector<int> writers(per, 0);
    for (int at = 0; at < per; at += 4) {
      const FourColumns f = four_columns(at, per);
      if (f.at < 0 || f.at + 4 > per || f.others < 0 || f.others > 3) return std::printf("per %d, at %d: columns %d .. of which %d are others'\n", per, at, f.at, f.others), 1;
      for (int e = f.others; e < 4; ++e) ++writers[f.at + e];
    }
    for (int c = 0; c < per; ++c)
      if (writers[c] != 1) return std::printf("per %d: column %d has %d writers\n", per, c, writers[c]), 1;
  }
  std::printf("four columns ok\n");
  return 0;
}
