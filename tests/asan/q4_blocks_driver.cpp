// Host program: the metadata check with blocks that hold nothing.
#include <stdio.h>

#include "../../paper_2608_04074_amd/csrc/host_checks.h"

using namespace novakv::host;

static int bad = 0;
static void expect(const char *what, nova_kv_status got, nova_kv_status want) {
  if (got == want) return;
  fprintf(stderr, "%s: status %d, expected %d (%s)\n", what, got, want, nova_kv_last_error());
  ++bad;
}

int main() {
  int32_t table[] = {3, -1, 1, 4, 5, -2147483647 - 1};
  const nova_kv_layout lay{16, 3, table};
  const int32_t lens[] = {48, 40}, start[] = {14, 44}, clash[] = {0, 10};
  expect("reads, blocks required", check_metadata(&lay, 6, 2, lens, 48, nullptr, 0), NOVA_KV_ERR_INVALID_ARG);
  expect("reads", check_metadata(&lay, 6, 2, lens, 48, nullptr, 0, nullptr, true), NOVA_KV_OK);
  expect("writes, blocks required", check_metadata(&lay, 6, 2, nullptr, 0, start, 4), NOVA_KV_ERR_INVALID_ARG);
  expect("writes", check_metadata(&lay, 6, 2, nullptr, 0, start, 4, nullptr, true), NOVA_KV_OK);
  table[3] = 6;
  expect("past the pool", check_metadata(&lay, 6, 2, lens, 48, nullptr, 0, nullptr, true), NOVA_KV_ERR_INVALID_ARG);
  table[3] = 3;
  expect("the same row", check_metadata(&lay, 6, 2, nullptr, 0, clash, 12, nullptr, true), NOVA_KV_ERR_INVALID_ARG);
  return bad != 0;
}
