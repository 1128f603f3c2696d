// Host program for the sanitizer test of the host check of the blocks that several query tokens
// attend: fixed cases, then random ones against a walk over positions.
#include <stdio.h>

#include <random>
#include <vector>

#include "../../paper_2608_04074_amd/csrc/host_checks.h"

using namespace novakv::host;

static int bad = 0;
static void expect(const char *what, nova_kv_status got, nova_kv_status want) {
  if (got != want) {
    fprintf(stderr, "%s: status %d, expected %d (%s)\n", what, got, want, nova_kv_last_error());
    ++bad;
  }
}

int main() {
  const nova_kv_status kBad = NOVA_KV_ERR_INVALID_ARG;
  // the blocks in front of a window are released, and the last one, which only a band holds
  const int32_t table[8] = {-5, -5, 2, 7, 0, 1, 3, 1 << 30};
  const nova_kv_layout lay{16, 4, table};
  const nova_kv_band band{4, 20, nullptr, nullptr}, recent{0, 20, nullptr, nullptr};
  int32_t sizes[2] = {60, 64}, counts[2] = {4, 2};
  auto check = [&](int first, int batch, int window, const nova_kv_band *b, int blocks = 8) {
    const nova_kv_layout own{16, 4, table + 4 * first};
    return check_attended(&own, blocks, batch, 4, counts + first, sizes + first, 64, window, b);
  };
  expect("released in front of the window", check(0, 1, 25, nullptr), NOVA_KV_OK);
  expect("the window reaches a released block", check(0, 1, 26, nullptr), kBad);
  expect("no window", check(0, 1, 0, nullptr), kBad);
  expect("sinks of a band do not cover a block", check(0, 1, 0, &band), kBad);
  expect("past the pool", check(0, 1, 25, nullptr, 7), kBad);
  expect("an unknown number of blocks", check(0, 1, 25, nullptr, 0), NOVA_KV_OK);
  expect("a block of the band only", check(1, 1, 0, &recent), NOVA_KV_OK);
  expect("without the band", check(1, 1, 0, nullptr), kBad);
  counts[0] = 0;
  expect("no queries", check(0, 1, 0, nullptr), NOVA_KV_OK);
  counts[0] = -7;
  expect("fewer than none", check(0, 1, 0, nullptr), NOVA_KV_OK);
  counts[0] = 1;
  expect("one query sees less than four do", check(0, 1, 28, nullptr), NOVA_KV_OK);
  sizes[0] = 65;
  expect("a length past the bound", check(0, 1, 25, nullptr), kBad);
  sizes[0] = -1;
  expect("a negative length", check(0, 1, 25, nullptr), kBad);

  std::mt19937_64 rng(1);
  for (int i = 0; i < 20000; ++i) {
    const int bs = 1 + static_cast<int>(rng() % 20), bps = 1 + static_cast<int>(rng() % 6), cap = bs * bps, batch = 1 + static_cast<int>(rng() % 2);
    std::vector<int32_t> t(batch * bps), size(batch), count(batch);
    for (auto &x : t) x = static_cast<int32_t>(rng() % 12) - 2;
    for (auto &x : size) x = static_cast<int32_t>(rng() % (cap + 1));
    for (auto &x : count) x = rng() % 8 ? static_cast<int32_t>(rng() % 12) - 2 : static_cast<int32_t>(rng());
    const int n = static_cast<int>(rng() % 10), window = rng() % 2 ? static_cast<int>(rng() % (cap + 1)) : 0;
    const bool banded = rng() & 1, given = rng() & 1;
    const nova_kv_band b{static_cast<int32_t>(rng() % 10), static_cast<int32_t>(rng() % 20), nullptr, nullptr};
    bool fine = true;
    for (int s = 0; s < batch; ++s) {
      const int m = given ? std::max(0, std::min(count[s], n)) : n;
      for (int x = 0; x < m; ++x) {
        const int p = size[s] - m + x;
        for (int j = 0; j <= p; ++j) {
          if (window > 0 && j <= p - window) continue;
          if (banded && (j < b.n_sink || j >= size[s] - b.n_rec)) continue;
          const int block = t[s * bps + j / bs];
          fine = fine && block >= 0 && block < 9;
        }
      }
    }
    const nova_kv_layout own{bs, bps, t.data()};
    const nova_kv_status got = check_attended(&own, 9, batch, n, given ? count.data() : nullptr, size.data(), cap, window, banded ? &b : nullptr);
    expect("random", got, fine ? NOVA_KV_OK : kBad);
  }
  return bad != 0;
}
