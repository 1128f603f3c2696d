// Host program for the sanitizer test of the host checks of positions on several axes and of the
// calls that read a cache back: fixed cases, then random ones whose arithmetic must not overflow.
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

static const void *at(uintptr_t x) { return reinterpret_cast<const void *>(x); }

int main() {
  const nova_kv_status kBad = NOVA_KV_ERR_INVALID_ARG;
  nova_kv_rotary r{};
  r.rotary_dim = 128;
  const int32_t some = 0;
  nova_kv_axes axes{3, {}};
  expect("axes", check_axes(&axes, &r, &some), NOVA_KV_OK);
  axes.pair_axis[63] = 3;
  expect("a pair without an axis", check_axes(&axes, &r, &some), kBad);
  r.rotary_dim = 64;
  expect("pairs that are not rotated", check_axes(&axes, &r, &some), NOVA_KV_OK);
  axes.num_axes = 5;
  expect("five axes", check_axes(&axes, &r, &some), kBad);

  expect("rows", check_read_outputs(NOVA_KV_BF16, 2, 10, 8, 128, at(1 << 20), at((1 << 20) + 2 * 10 * 8 * 128 * 2)), NOVA_KV_OK);
  expect("rows that overlap", check_read_outputs(NOVA_KV_F32, 2, 10, 8, 128, at(1 << 20), at((1 << 20) + 2 * 10 * 8 * 128 * 2)), kBad);
  expect("one side", check_read_outputs(NOVA_KV_F32, 2, 10, 8, 128, nullptr, at(1 << 20)), NOVA_KV_OK);
  expect("too many", check_read_outputs(NOVA_KV_F32, 65535, 0x7fffffff, 8, 128, nullptr, at(1 << 20)), NOVA_KV_ERR_UNSUPPORTED);

  // two sequences that share block 1; the last block of the second is held by a band only
  const int32_t table[6] = {0, 1, 2, 1, 3, -1}, sizes[2] = {40, 48}, lens[2] = {30, 100};
  const nova_kv_layout lay{16, 3, table};
  const nova_kv_band band{2, 16, nullptr, nullptr};
  int32_t start[2] = {0, 0};
  expect("shared blocks", check_reads(&lay, 4, 2, start, 32, nullptr, sizes, nullptr, false), NOVA_KV_OK);
  expect("a released block", check_reads(&lay, 4, 2, start, 40, nullptr, sizes, nullptr, false), kBad);
  expect("a released block, may be absent", check_reads(&lay, 4, 2, start, 40, nullptr, sizes, nullptr, true), NOVA_KV_OK);
  expect("a released block behind the band", check_reads(&lay, 4, 2, start, 48, lens, sizes, &band, false), NOVA_KV_OK);
  expect("past the pool", check_reads(&lay, 3, 2, start, 32, nullptr, sizes, nullptr, false), kBad);
  start[0] = 20;
  expect("past the length", check_reads(&lay, 4, 2, start, 21, nullptr, sizes, nullptr, true), kBad);
  expect("nothing past the length", check_reads(&lay, 4, 1, start, 0, nullptr, sizes, nullptr, true), NOVA_KV_OK);
  start[0] = -1;
  expect("in front", check_reads(&lay, 4, 2, start, 4, nullptr, sizes, nullptr, true), kBad);

  std::mt19937_64 rng(1);
  for (int i = 0; i < 20000; ++i) {  // any status, no overflow, no read past the arrays
    nova_kv_axes x{};
    x.num_axes = static_cast<int32_t>(rng() % 7) - 1;
    for (auto &p : x.pair_axis) p = static_cast<uint8_t>(rng() % 5);
    r.rotary_dim = 8 * static_cast<int32_t>(rng() % 17);
    (void)check_axes(&x, &r, &some);
    (void)check_read_outputs(static_cast<nova_kv_dtype>(rng() % 3), static_cast<int32_t>(rng()), static_cast<int32_t>(rng()),
                             1 + static_cast<int32_t>(rng() % 0x7fffffff), 128, at(16 * (rng() >> 8)), at(16 * (rng() >> 8)));
    int32_t starts[2], counts[2], held[2];
    for (int b = 0; b < 2; ++b)
      starts[b] = static_cast<int32_t>(rng() >> (rng() % 64)), counts[b] = static_cast<int32_t>(rng() >> (rng() % 64)),
      held[b] = static_cast<int32_t>(rng() % 60);
    (void)check_reads(&lay, static_cast<int32_t>(rng() % 6), 2, starts, static_cast<int32_t>(rng() & 0x7fffffff), rng() & 1 ? counts : nullptr,
                      rng() & 1 ? held : nullptr, nullptr, rng() & 1);
  }
  return bad != 0;
}
