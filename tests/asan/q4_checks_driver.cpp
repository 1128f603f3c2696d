// Host program for the sanitizer test of the host checks of the norm, rotation
// and 4-bit cache calls: fixed cases of the argument checks, then random ones
// whose arithmetic on strides, sizes and addresses must not overflow, and the
// metadata check with sequences that write fewer tokens than the call's.
#include <stdio.h>
#include <stdlib.h>

#include <random>

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
  nova_kv_rotary r{};
  r.num_q_heads = 32;
  r.num_kv_heads = 8;
  r.head_dim = 128;
  r.rotary_dim = 64;
  r.num_positions = 100;
  r.cos_sin = static_cast<const float *>(at(4096));
  r.eps = 1e-6f;
  expect("rotary", check_rotary(&r, true, true), NOVA_KV_OK);
  expect("rotary null", check_rotary(nullptr, true, true), NOVA_KV_ERR_INVALID_ARG);
  r.q_norm = static_cast<const float *>(at(4100));
  expect("odd weights", check_rotary(&r, true, false), NOVA_KV_ERR_INVALID_ARG);
  expect("odd weights of an absent side", check_rotary(&r, false, true), NOVA_KV_OK);
  nova_kv_q4_cache c{8, 128, 0x7fffffff, {16, 16, nullptr}, (uint8_t *)at(1 << 20), (uint8_t *)at(2 << 20), (uint16_t *)at(3 << 20),
                     (uint16_t *)at(4 << 20)};
  expect("a pool of too many rows", check_q4_cache(&c), NOVA_KV_ERR_UNSUPPORTED);
  c.layout.block_size = 1 << 15, c.layout.blocks_per_seq = 1 << 15;
  expect("rows past 2^45", check_q4_cache(&c), NOVA_KV_ERR_UNSUPPORTED);
  c.num_blocks = 4;
  expect("a cache", check_q4_cache(&c), NOVA_KV_OK);

  // an output over its own dense input only
  const nova_kv_rows dense{at(1 << 20), 4 * 4096, 4096}, strided{at(1 << 20), 4 * 8192, 8192};
  expect("in place", check_overlaps(&r, &dense, nullptr, nullptr, NOVA_KV_BF16, 2, 4, at(1 << 20), nullptr, nullptr), NOVA_KV_OK);
  expect("in place, strided", check_overlaps(&r, &strided, nullptr, nullptr, NOVA_KV_BF16, 2, 4, at(1 << 20), nullptr, nullptr),
         NOVA_KV_ERR_INVALID_ARG);
  expect("one token, any stride", check_overlaps(&r, &strided, nullptr, nullptr, NOVA_KV_BF16, 1, 1, at(1 << 20), nullptr, nullptr),
         NOVA_KV_OK);
  expect("next to it", check_overlaps(&r, &dense, nullptr, nullptr, NOVA_KV_BF16, 2, 4, at((1 << 20) + 2 * 4 * 4096 * 2), nullptr, nullptr),
         NOVA_KV_OK);

  std::mt19937_64 rng(1);
  auto pick = [&](uint64_t n) { return rng() % n; };
  for (int i = 0; i < 20000; ++i) {  // extreme sizes, strides and addresses: any status, no overflow
    nova_kv_rotary x{};
    x.num_q_heads = static_cast<int32_t>(rng());
    x.num_kv_heads = static_cast<int32_t>(rng());
    x.head_dim = pick(2) ? 128 : static_cast<int32_t>(rng());
    x.rotary_dim = static_cast<int32_t>(rng());
    (void)check_rotary(&x, true, true);
    nova_kv_q4_cache y{static_cast<int32_t>(rng()), pick(2) ? 64 : 128, static_cast<int32_t>(rng()),
                       {static_cast<int32_t>(rng()), static_cast<int32_t>(rng()), nullptr}, nullptr, nullptr, nullptr, nullptr};
    (void)check_q4_cache(&y);
    x.num_q_heads = 1 + pick(1 << 16), x.num_kv_heads = 1 + pick(1 << 16), x.head_dim = 128;
    nova_kv_rows rows[3];
    for (auto &q : rows) {
      q.data = at(rng());
      q.batch_stride = pick((1ull << 40) + 1);
      q.token_stride = pick((1ull << 40) + 1);
      (void)check_rows("x", &q, at(rng()), pick(2) ? NOVA_KV_BF16 : NOVA_KV_F32, pick(2));
    }
    (void)check_overlaps(&x, &rows[0], &rows[1], &rows[2], NOVA_KV_F32, 1 + pick(65535), 1 + pick(0x7fffffff), at(rng()), at(rng()),
                         at(rng()));
  }

  // new_lens: only the positions that a sequence writes must lie in the cache
  int32_t *start = static_cast<int32_t *>(malloc(2 * sizeof(int32_t))), *lens = static_cast<int32_t *>(malloc(2 * sizeof(int32_t)));
  start[0] = 0, start[1] = 30;
  const nova_kv_layout lay{16, 2, nullptr};
  expect("past the capacity", check_metadata(&lay, 4, 2, nullptr, 0, start, 4), NOVA_KV_ERR_INVALID_ARG);
  lens[0] = 4, lens[1] = 2;
  expect("two of four tokens", check_metadata(&lay, 4, 2, nullptr, 0, start, 4, lens), NOVA_KV_OK);
  lens[1] = 3;
  expect("three of four tokens", check_metadata(&lay, 4, 2, nullptr, 0, start, 4, lens), NOVA_KV_ERR_INVALID_ARG);
  lens[0] = 99, lens[1] = -7;
  expect("lengths are cut", check_metadata(&lay, 4, 2, nullptr, 0, start, 4, lens), NOVA_KV_OK);
  start[1] = -5;
  expect("nothing written", check_metadata(&lay, 4, 2, nullptr, 0, start, 4, lens), NOVA_KV_OK);
  free(start);
  free(lens);
  return bad != 0;
}
