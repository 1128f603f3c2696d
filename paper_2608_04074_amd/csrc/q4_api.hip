// C ABI of the norm and rotation of heads and of the cache held in 4 bits:
// host-side validation, workspace planning and dispatch.  Every check runs
// before any HIP call, so an invalid call launches nothing.
#include <math.h>

#include <exception>

#include "../../include/nova_kv.h"
#include "debug_check.h"
#include "host_checks.h"
#include "q4_internal.h"

using namespace novakv::host;

namespace {

// No exception leaves a C entry (the debug mode's host copies may throw).
template <typename F>
nova_kv_status guarded(F f) {
  try {
    return f();
  } catch (const std::exception &e) {
    return fail(NOVA_KV_ERR_HIP, "host: %s", e.what());
  }
}

// The rows of a unit and the threads of a launch (768 a tile) are counted in 32 bits.
bool too_many_rows(int32_t batch, int32_t n_q, int32_t num_q_heads, int32_t num_kv_heads) {
  const long long rows = static_cast<long long>(n_q) * (num_q_heads / num_kv_heads);
  return batch > 65535 || rows > (1 << 24) || ((rows + 15) / 16) * num_kv_heads > (1 << 22) / batch;
}

novakv::HeadRows to_rows(const nova_kv_rows *r) {
  return r ? novakv::HeadRows{r->data, r->batch_stride, r->token_stride} : novakv::HeadRows{nullptr, 0, 0};
}

// What both calls check of their tokens.
nova_kv_status check_tokens(const nova_kv_rotary *r, nova_kv_dtype dtype, int32_t batch, int32_t n_new) {
  if (dtype != NOVA_KV_F32 && dtype != NOVA_KV_BF16)
    return fail(NOVA_KV_ERR_INVALID_ARG, "dtype must be NOVA_KV_F32 or NOVA_KV_BF16");
  if (batch < 0 || n_new < 0) return fail(NOVA_KV_ERR_INVALID_ARG, "batch and n_new must be >= 0");
  if (batch > 65535) return fail(NOVA_KV_ERR_INVALID_ARG, "batch > 65535");
  if (static_cast<long long>(batch) * n_new >= (1LL << 24))  // a launch's threads: 256 a token
    return fail(NOVA_KV_ERR_UNSUPPORTED, "more than 2^24 - 1 tokens in a call");
  return NOVA_KV_OK;
}

novakv::RotateArgs rotate_args(const nova_kv_rotary *r, const nova_kv_rows *q, const nova_kv_rows *k,
                               const nova_kv_rows *v, nova_kv_dtype dtype, int32_t batch, int32_t n_new,
                               const int32_t *new_lens, const int32_t *start_pos) {
  novakv::RotateArgs a{};
  a.batch = batch;
  a.n_new = n_new;
  a.head_dim = r->head_dim;
  a.nq = q ? r->num_q_heads : 0;
  a.nk = k ? r->num_kv_heads : 0;
  a.nv = v ? r->num_kv_heads : 0;
  a.bf16 = dtype == NOVA_KV_BF16;
  a.q = to_rows(q);
  a.k = to_rows(k);
  a.v = to_rows(v);
  a.new_lens = new_lens;
  a.start_pos = start_pos;
  a.cos_sin = r->rotary_dim ? r->cos_sin : nullptr;
  a.rotary_dim = r->rotary_dim;
  a.interleaved = r->interleaved;
  a.num_positions = r->num_positions;
  a.q_norm = r->q_norm;
  a.k_norm = r->k_norm;
  a.q_norm_stride = r->q_norm_per_head ? r->head_dim : 0;
  a.k_norm_stride = r->k_norm_per_head ? r->head_dim : 0;
  a.eps = r->eps;
  return a;
}

}  // namespace

extern "C" {

nova_kv_status nova_kv_rotate_qkv(const nova_kv_rotary *r, const nova_kv_rows *q, const nova_kv_rows *k,
                                  const nova_kv_rows *v, nova_kv_dtype dtype, int32_t batch, int32_t n_new,
                                  const int32_t *new_lens, const int32_t *start_pos, void *q_out, void *k_out,
                                  void *v_out, void *hip_stream) {
  nova_kv_status st = check_rotary(r, q != nullptr, k != nullptr);
  if (st != NOVA_KV_OK) return st;
  if ((st = check_tokens(r, dtype, batch, n_new)) != NOVA_KV_OK) return st;
  if (batch == 0 || n_new == 0) return ok();
  if ((st = check_rows("q", q, q_out, dtype, true)) != NOVA_KV_OK) return st;
  if ((st = check_rows("k", k, k_out, dtype, true)) != NOVA_KV_OK) return st;
  if ((st = check_rows("v", v, v_out, dtype, true)) != NOVA_KV_OK) return st;
  if (!q && !k && !v) return ok();
  if ((st = check_overlaps(r, q, k, v, dtype, batch, n_new, q_out, k_out, v_out)) != NOVA_KV_OK) return st;
  if (r->rotary_dim && !start_pos) return fail(NOVA_KV_ERR_INVALID_ARG, "start_pos is NULL");
  novakv::RotateArgs a = rotate_args(r, q, k, v, dtype, batch, n_new, new_lens, start_pos);
  a.q_out = q_out;
  a.k_out = k_out;
  a.v_out = v_out;
  const hipError_t e = novakv::launch_rotate(a, static_cast<hipStream_t>(hip_stream));
  if (e != hipSuccess) return fail(NOVA_KV_ERR_HIP, "rotate launch: %s", hipGetErrorString(e));
  return ok();
}

nova_kv_status nova_kv_q4_append(const nova_kv_rotary *r, const nova_kv_q4_cache *cache, const nova_kv_rows *q,
                                 const nova_kv_rows *k, const nova_kv_rows *v, nova_kv_dtype dtype, int32_t batch,
                                 int32_t n_new, const int32_t *new_lens, const int32_t *start_pos, void *q_out,
                                 void *k_held, void *v_held, void *hip_stream) {
  return guarded([&]() -> nova_kv_status {
    nova_kv_status st = check_rotary(r, q != nullptr, true);
    if (st != NOVA_KV_OK) return st;
    if ((st = check_q4_cache(cache)) != NOVA_KV_OK) return st;
    if (cache->num_kv_heads != r->num_kv_heads || cache->head_dim != r->head_dim)
      return fail(NOVA_KV_ERR_INVALID_ARG, "the cache holds %d heads of %d, rotary says %d of %d", cache->num_kv_heads,
                  cache->head_dim, r->num_kv_heads, r->head_dim);
    if ((st = check_tokens(r, dtype, batch, n_new)) != NOVA_KV_OK) return st;
    if (batch == 0 || n_new == 0) return ok();
    if (!k || !v) return fail(NOVA_KV_ERR_INVALID_ARG, "k or v is NULL");
    if ((st = check_rows("q", q, q_out, dtype, true)) != NOVA_KV_OK) return st;
    if ((st = check_rows("k", k, k_held, dtype, false)) != NOVA_KV_OK) return st;
    if ((st = check_rows("v", v, v_held, dtype, false)) != NOVA_KV_OK) return st;
    if ((st = check_overlaps(r, q, k, v, dtype, batch, n_new, q_out, k_held, v_held)) != NOVA_KV_OK) return st;
    if (!start_pos) return fail(NOVA_KV_ERR_INVALID_ARG, "start_pos is NULL");
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if ((st = novakv::debug_check(&cache->layout, batch, nullptr, 0, start_pos, n_new, stream, new_lens,
                                  cache->num_blocks)) != NOVA_KV_OK)
      return st;
    novakv::RotateArgs a = rotate_args(r, q, k, v, dtype, batch, n_new, new_lens, start_pos);
    a.q_out = q_out;
    a.k_out = k_held;
    a.v_out = v_held;
    a.q4 = 1;
    a.layout = novakv::CacheLayout{cache->layout.block_size, cache->layout.blocks_per_seq, cache->layout.block_table};
    a.num_blocks = cache->num_blocks;
    a.k_codes = cache->k_codes;
    a.v_codes = cache->v_codes;
    a.k_sq = cache->k_sq;
    a.v_sq = cache->v_sq;
    const hipError_t e = novakv::launch_rotate(a, stream);
    if (e != hipSuccess) return fail(NOVA_KV_ERR_HIP, "4-bit append launch: %s", hipGetErrorString(e));
    return ok();
  });
}

size_t nova_kv_q4_attn_workspace_bytes(const nova_kv_q4_cache *cache, int32_t batch, int32_t n_q, int32_t num_q_heads,
                                       int32_t max_seq_len) {
  if (!cache || batch <= 0 || n_q <= 0 || num_q_heads <= 0 || max_seq_len <= 0 || max_seq_len > (1 << 30) ||
      cache->num_kv_heads <= 0 || (cache->head_dim != 64 && cache->head_dim != 128) || num_q_heads % cache->num_kv_heads != 0 ||
      too_many_rows(batch, n_q, num_q_heads, cache->num_kv_heads))
    return 0;
  return novakv::plan_q4_attn(batch, n_q, num_q_heads, cache->num_kv_heads, cache->head_dim, 1, max_seq_len, 0).total;
}

nova_kv_status nova_kv_q4_attn(const nova_kv_q4_cache *cache, const void *q, nova_kv_dtype q_dtype, int32_t batch,
                               int32_t n_q, int32_t num_q_heads, const int32_t *q_lens, const int32_t *seq_lens,
                               int32_t max_seq_len, int32_t window, const float *sinks, float softmax_scale,
                               void *out, void *workspace, size_t workspace_bytes, void *hip_stream) {
  return guarded([&]() -> nova_kv_status {
    nova_kv_status st = check_q4_cache(cache);
    if (st != NOVA_KV_OK) return st;
    if (q_dtype != NOVA_KV_F32 && q_dtype != NOVA_KV_BF16)
      return fail(NOVA_KV_ERR_INVALID_ARG, "q_dtype must be NOVA_KV_F32 or NOVA_KV_BF16");
    if (batch < 0 || n_q < 0) return fail(NOVA_KV_ERR_INVALID_ARG, "batch and n_q must be >= 0");
    if (batch > 65535) return fail(NOVA_KV_ERR_INVALID_ARG, "batch > 65535");
    if (num_q_heads <= 0 || num_q_heads % cache->num_kv_heads != 0)
      return fail(NOVA_KV_ERR_INVALID_ARG, "num_q_heads (%d) must be a positive multiple of num_kv_heads (%d)",
                  num_q_heads, cache->num_kv_heads);
    if (max_seq_len <= 0) return fail(NOVA_KV_ERR_INVALID_ARG, "max_seq_len must be > 0");
    if (static_cast<long long>(max_seq_len) >
        static_cast<long long>(cache->layout.block_size) * cache->layout.blocks_per_seq)
      return fail(NOVA_KV_ERR_INVALID_ARG, "max_seq_len exceeds the per-sequence capacity");
    if (window < 0) return fail(NOVA_KV_ERR_INVALID_ARG, "window must be >= 0");
    if (!(softmax_scale >= 0.f) || softmax_scale > 1e30f)
      return fail(NOVA_KV_ERR_INVALID_ARG, "softmax_scale must be in [0, 1e30]");
    if (batch == 0 || n_q == 0) return ok();
    if (!q || !seq_lens || !out) return fail(NOVA_KV_ERR_INVALID_ARG, "q, seq_lens or out is NULL");
    if (!aligned(q, 16) || !aligned(out, 16)) return fail(NOVA_KV_ERR_INVALID_ARG, "q and out must be 16-byte aligned");
    if (too_many_rows(batch, n_q, num_q_heads, cache->num_kv_heads))
      return fail(NOVA_KV_ERR_UNSUPPORTED, "too many query rows in a call");
    const novakv::Q4AttnPlan plan = novakv::plan_q4_attn(batch, n_q, num_q_heads, cache->num_kv_heads, cache->head_dim,
                                                         q_dtype == NOVA_KV_BF16, max_seq_len, window);
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if ((st = novakv::debug_check(&cache->layout, batch, seq_lens, max_seq_len, nullptr, 0, stream, nullptr,
                                  cache->num_blocks)) != NOVA_KV_OK)
      return st;
    if (plan.n_split > 1) {
      if (!workspace || workspace_bytes < plan.total)
        return fail(NOVA_KV_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", plan.total,
                    workspace ? workspace_bytes : static_cast<size_t>(0));
      if (!aligned(workspace, 256)) return fail(NOVA_KV_ERR_WORKSPACE, "workspace must be 256-byte aligned");
    }
    novakv::Q4AttnArgs a{};
    a.batch = batch;
    a.n_q = n_q;
    a.num_q_heads = num_q_heads;
    a.num_kv_heads = cache->num_kv_heads;
    a.head_dim = cache->head_dim;
    a.gqa = num_q_heads / cache->num_kv_heads;
    a.layout = novakv::CacheLayout{cache->layout.block_size, cache->layout.blocks_per_seq, cache->layout.block_table};
    a.num_blocks = cache->num_blocks;
    a.k_codes = cache->k_codes;
    a.v_codes = cache->v_codes;
    a.k_sq = cache->k_sq;
    a.v_sq = cache->v_sq;
    a.q = q;
    a.q_bf16 = q_dtype == NOVA_KV_BF16;
    a.q_lens = q_lens;
    a.seq_lens = seq_lens;
    a.max_seq_len = max_seq_len;
    a.window = window;
    a.sinks = sinks;
    a.qscale = (softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf(static_cast<float>(cache->head_dim))) *
               1.44269504088896341f;
    a.out = out;
    a.n_split = plan.n_split;
    a.row_tiles = plan.row_tiles;
    char *ws = static_cast<char *>(workspace);
    a.counters = plan.n_split > 1 ? reinterpret_cast<int *>(ws) : nullptr;
    a.part = plan.n_split > 1 ? reinterpret_cast<float *>(ws + plan.off_part) : nullptr;
    const hipError_t e = novakv::launch_q4_attn(a, plan, stream);
    if (e != hipSuccess) return fail(NOVA_KV_ERR_HIP, "4-bit attention launch: %s", hipGetErrorString(e));
    return ok();
  });
}

}  // extern "C"
