// Host program of the stores of rotated rows: where they may be streamed, the lanes of a store write whole
// lines of 64 bytes, and where they write parts of lines they may not.
#include <stdio.h>

#include <set>
#include <vector>

#include "../../paper_2608_04074_amd/csrc/rotate_layout.h"

using namespace novakv::rotate;

int main() {
  int bad = 0;
  for (int d : {64, 128})
    for (int r = 0; r <= d; r += 8)
      for (bool il : {false, true})
        for (bool bf16 : {false, true}) {
          const int elem = bf16 ? 2 : 4;
          // one store of the row's lanes: eight coordinates that follow each other in 16 bytes, or a chunk of four
          std::vector<std::set<int>> stores(il && bf16 ? 1 : 2);
          for (int lane = 0; lane < d / 8; ++lane) {
            const LaneChunks l = lane_chunks(lane, r, il);
            if (stores.size() == 1 && l.c1 != l.c0 + 4) ++bad;
            for (int j = 0; j < 4 * elem; ++j) stores.front().insert(l.c0 * elem + j), stores.back().insert(l.c1 * elem + j);
          }
          bool whole = true;
          for (const auto &bytes : stores)
            for (int x : bytes) {  // each byte's line
              int held = 0;
              for (int y : bytes) held += y / 64 == x / 64;
              whole = whole && held == 64;
            }
          if (whole_lines(d, r, il, bf16) && !whole) printf("head_dim %d rotary_dim %d interleaved %d bf16 %d\n", d, r, il, bf16), ++bad;
          if (il && !bf16 && (whole || whole_lines(d, r, il, bf16))) ++bad;
        }
  return bad != 0;
}
