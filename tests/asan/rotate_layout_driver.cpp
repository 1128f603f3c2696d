// Host program of the stores of a row's 4-bit codes: every coordinate is held once, every byte of the row is stored
// once, and every store is aligned to its width.
#include <stdio.h>

#include <vector>

#include "../../paper_2608_04074_amd/csrc/rotate_layout.h"

using namespace novakv::rotate;

int main() {
  int bad = 0;
  for (int d : {64, 128})
    for (int r = 0; r <= d; r += 8)
      for (bool il : {false, true}) {
        std::vector<int> held(d), stored(d / 2);
        for (int lane = 0; lane < d / 8; ++lane) {
          const LaneChunks l = lane_chunks(lane, r, il);
          for (int j = 0; j < 4; ++j) ++held.at(l.c0 + j), ++held.at(l.c1 + j);
          const CodeStore how = code_store(l, r, il);
          auto store = [&](int at, int bytes) {
            if (at % bytes) printf("head_dim %d rotary_dim %d interleaved %d lane %d: %d bytes at byte %d\n", d, r, il, lane, bytes, at), ++bad;
            for (int j = 0; j < bytes; ++j) ++stored.at(at + j);
          };
          if (how == CodeStore::kApart) store(l.c0 / 2, 2), store(l.c1 / 2, 2);
          else store(word_at(l, how, lane), 4);
          // who exchanges has a partner that does too
          if (how == CodeStore::kExchange && code_store(lane_chunks(lane ^ 1, r, il), r, il) != how) ++bad;
        }
        for (int x : held) bad += x != 1;
        for (int x : stored) bad += x != 1;
      }
  return bad != 0;
}
