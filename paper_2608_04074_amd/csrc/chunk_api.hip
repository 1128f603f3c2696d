// C ABI of the attention of several query tokens over the 2-bit cache and of reading that cache
// back: host-side validation and dispatch.  Every check runs before any HIP call, so an invalid
// call launches nothing.
#include <math.h>

#include <exception>

#include "../../include/nova_kv.h"
#include "chunk_internal.h"
#include "debug_check.h"
#include "host_checks.h"

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

// The rows of a unit and the threads of a launch (512 a tile) are counted in 32 bits.
bool too_many_rows(int32_t batch, int32_t n_q, int32_t num_q_heads, int32_t num_kv_heads) {
  const long long rows = static_cast<long long>(n_q) * (num_q_heads / num_kv_heads);
  return batch > 65535 || rows > (1 << 24) || ((rows + 15) / 16) * num_kv_heads > (1 << 22) / batch;
}

}  // namespace

extern "C" {

size_t nova_kv_chunk_attn_workspace_bytes(const nova_kv_params *p, int32_t batch, int32_t n_q, int32_t num_q_heads,
                                          int32_t max_seq_len) {
  if (!p || batch <= 0 || n_q <= 0 || num_q_heads <= 0 || max_seq_len <= 0 || max_seq_len > (1 << 30) || p->num_kv_heads <= 0 ||
      (p->head_dim != 64 && p->head_dim != 128) || num_q_heads % p->num_kv_heads != 0 ||
      too_many_rows(batch, n_q, num_q_heads, p->num_kv_heads))
    return 0;
  return novakv::plan_chunk(batch, n_q, num_q_heads, p->num_kv_heads, p->head_dim, max_seq_len, 0).total;
}

nova_kv_status nova_kv_chunk_attn(const nova_kv_params *p, const nova_kv_layout *layout, const void *q,
                                  nova_kv_dtype q_dtype, int32_t batch, int32_t n_q, int32_t num_q_heads,
                                  const int32_t *q_lens, const uint8_t *k_codes, const uint8_t *v_codes,
                                  const uint16_t *k_scales, const uint16_t *v_sq, const nova_kv_band *band,
                                  const int32_t *seq_lens, int32_t max_seq_len, int32_t window, const float *sinks,
                                  float softmax_scale, void *out, void *workspace, size_t workspace_bytes,
                                  void *hip_stream) {
  return guarded([&]() -> nova_kv_status {
    nova_kv_status st = check_params(p, false, true);
    if (st != NOVA_KV_OK) return st;
    if ((st = check_layout(layout)) != NOVA_KV_OK) return st;
    if (q_dtype != NOVA_KV_F32 && q_dtype != NOVA_KV_BF16)
      return fail(NOVA_KV_ERR_INVALID_ARG, "q_dtype must be NOVA_KV_F32 or NOVA_KV_BF16");
    if (batch < 0 || n_q < 0) return fail(NOVA_KV_ERR_INVALID_ARG, "batch and n_q must be >= 0");
    if (batch > 65535) return fail(NOVA_KV_ERR_INVALID_ARG, "batch > 65535");
    if (num_q_heads <= 0 || num_q_heads % p->num_kv_heads != 0)
      return fail(NOVA_KV_ERR_INVALID_ARG, "num_q_heads (%d) must be a positive multiple of num_kv_heads (%d)", num_q_heads,
                  p->num_kv_heads);
    if (max_seq_len <= 0) return fail(NOVA_KV_ERR_INVALID_ARG, "max_seq_len must be > 0");
    if (static_cast<long long>(max_seq_len) > static_cast<long long>(layout->block_size) * layout->blocks_per_seq)
      return fail(NOVA_KV_ERR_INVALID_ARG, "max_seq_len exceeds the per-sequence capacity");
    if (window < 0) return fail(NOVA_KV_ERR_INVALID_ARG, "window must be >= 0");
    window = window_within(window, max_seq_len);
    if (!(softmax_scale >= 0.f) || softmax_scale > 1e30f)
      return fail(NOVA_KV_ERR_INVALID_ARG, "softmax_scale must be in [0, 1e30]");
    if (batch == 0 || n_q == 0) return ok();
    if ((st = check_scales(p, k_scales)) != NOVA_KV_OK) return st;
    if ((st = check_sq(p, v_sq)) != NOVA_KV_OK) return st;
    if ((st = check_band(band)) != NOVA_KV_OK) return st;
    if (!q || !k_codes || !v_codes || !seq_lens || !out)
      return fail(NOVA_KV_ERR_INVALID_ARG, "q, k_codes, v_codes, seq_lens or out is NULL");
    if (!aligned(q, 16) || !aligned(out, 16)) return fail(NOVA_KV_ERR_INVALID_ARG, "q and out must be 16-byte aligned");
    if (!aligned(k_codes, 16) || !aligned(v_codes, 16))
      return fail(NOVA_KV_ERR_INVALID_ARG, "code pools must be 16-byte aligned");
    if (too_many_rows(batch, n_q, num_q_heads, p->num_kv_heads))
      return fail(NOVA_KV_ERR_UNSUPPORTED, "too many query rows in a call");
    const novakv::ChunkPlan plan = novakv::plan_chunk(batch, n_q, num_q_heads, p->num_kv_heads, p->head_dim, max_seq_len, window);
    if (plan.n_split > 1) {
      if (!workspace || workspace_bytes < plan.total)
        return fail(NOVA_KV_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", plan.total,
                    workspace ? workspace_bytes : static_cast<size_t>(0));
      if (!aligned(workspace, 256)) return fail(NOVA_KV_ERR_WORKSPACE, "workspace must be 256-byte aligned");
    }
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if ((st = novakv::debug_check_attended(layout, batch, n_q, q_lens, seq_lens, max_seq_len, window, band, stream)) != NOVA_KV_OK)
      return st;
    novakv::ChunkArgs a{};
    a.batch = batch;
    a.n_q = n_q;
    a.num_q_heads = num_q_heads;
    a.num_kv_heads = p->num_kv_heads;
    a.head_dim = p->head_dim;
    a.gqa = num_q_heads / p->num_kv_heads;
    a.layout = novakv::CacheLayout{layout->block_size, layout->blocks_per_seq, layout->block_table};
    a.k_codes = k_codes;
    a.block_of.set(static_cast<uint32_t>(layout->block_size));
    a.v_codes = v_codes;
    a.v_sq = (p->flags & NOVA_KV_SQ_VALUES) ? v_sq : nullptr;
    a.q = q;
    a.q_bf16 = q_dtype == NOVA_KV_BF16;
    a.q_lens = q_lens;
    a.seq_lens = seq_lens;
    a.max_seq_len = max_seq_len;
    a.window = window;
    a.sinks = sinks;
    a.qscale = (softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf(static_cast<float>(p->head_dim))) * 1.44269504088896341f;
    a.out = out;
    a.n_split = plan.n_split;
    a.row_tiles = plan.row_tiles;
    char *ws = static_cast<char *>(workspace);
    a.counters = plan.n_split > 1 ? reinterpret_cast<int *>(ws) : nullptr;
    a.part = plan.n_split > 1 ? reinterpret_cast<float *>(ws + plan.off_part) : nullptr;
    a.kbar = p->kbar;
    a.t_k_inv_t = p->t_k_inv_t;
    a.t_v = p->t_v;
    a.cb_k = p->cb_k;
    a.cb_v = p->cb_v;
    a.t_bf16 = (p->flags & NOVA_KV_BF16_TRANSFORMS) ? 1 : 0;
    a.cb_fp8 = (p->flags & NOVA_KV_FP8_CODEBOOKS) ? 1 : 0;
    a.k_scales = (p->flags & NOVA_KV_KEY_SCALE) ? k_scales : nullptr;
    if (band) {
      a.n_sink = band->n_sink;
      a.n_rec = band->n_rec;
      a.band_k = band->k;
      a.band_v = band->v;
    }
    const hipError_t e = novakv::launch_chunk(a, plan, stream);
    if (e != hipSuccess) return fail(NOVA_KV_ERR_HIP, "chunk attention launch: %s", hipGetErrorString(e));
    return ok();
  });
}

nova_kv_status nova_kv_read(const nova_kv_params *p, const nova_kv_layout *layout, const uint8_t *k_codes,
                            const uint8_t *v_codes, const uint16_t *k_scales, const uint16_t *v_sq,
                            const nova_kv_band *band, const int32_t *seq_lens, nova_kv_dtype dtype, int32_t batch,
                            int32_t n, const int32_t *start_pos, const int32_t *lens, void *k_out, void *v_out,
                            void *hip_stream) {
  return guarded([&]() -> nova_kv_status {
    nova_kv_status st = check_params(p, false, true);
    if (st != NOVA_KV_OK) return st;
    if ((st = check_layout(layout)) != NOVA_KV_OK) return st;
    if ((st = check_read_outputs(dtype, batch, n, p->num_kv_heads, p->head_dim, k_out, v_out)) != NOVA_KV_OK) return st;
    if (batch == 0 || n == 0 || (!k_out && !v_out)) return ok();
    if (p->num_kv_heads > 4096) return fail(NOVA_KV_ERR_UNSUPPORTED, "num_kv_heads > 4096");  // a round's rows: 31 bits of bytes
    if (k_out && (st = check_scales(p, k_scales)) != NOVA_KV_OK) return st;
    if (v_out && (st = check_sq(p, v_sq)) != NOVA_KV_OK) return st;
    if ((st = check_band(band)) != NOVA_KV_OK) return st;
    if (!start_pos || (k_out && !k_codes) || (v_out && !v_codes))
      return fail(NOVA_KV_ERR_INVALID_ARG, "start_pos or a code pool is NULL");
    if (!aligned(k_codes, 16) || !aligned(v_codes, 16))
      return fail(NOVA_KV_ERR_INVALID_ARG, "code pools must be 16-byte aligned");
    if (band && !seq_lens) return fail(NOVA_KV_ERR_INVALID_ARG, "a band needs seq_lens");
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if ((st = novakv::debug_check_reads(layout, batch, start_pos, n, lens, seq_lens, band, stream)) != NOVA_KV_OK) return st;
    novakv::ReadArgs a{};
    a.batch = batch;
    a.n = n;
    a.num_kv_heads = p->num_kv_heads;
    a.head_dim = p->head_dim;
    a.layout = novakv::CacheLayout{layout->block_size, layout->blocks_per_seq, layout->block_table};
    a.lens = lens;
    a.start_pos = start_pos;
    a.seq_lens = seq_lens;
    a.k_out = k_out;
    a.v_out = v_out;
    a.bf16 = dtype == NOVA_KV_BF16;
    a.k_codes = k_codes;
    a.v_codes = v_codes;
    a.kbar = p->kbar;
    a.t_k_inv_t = p->t_k_inv_t;
    a.t_v = p->t_v;
    a.cb_k = p->cb_k;
    a.cb_v = p->cb_v;
    a.t_bf16 = (p->flags & NOVA_KV_BF16_TRANSFORMS) ? 1 : 0;
    a.cb_fp8 = (p->flags & NOVA_KV_FP8_CODEBOOKS) ? 1 : 0;
    a.k_scales = (p->flags & NOVA_KV_KEY_SCALE) ? k_scales : nullptr;
    a.v_sq = (p->flags & NOVA_KV_SQ_VALUES) ? v_sq : nullptr;
    if (band) {
      a.n_sink = band->n_sink;
      a.n_rec = band->n_rec;
      a.band_k = band->k;
      a.band_v = band->v;
    }
    const hipError_t e = novakv::launch_read(a, stream);
    if (e != hipSuccess) return fail(NOVA_KV_ERR_HIP, "read launch: %s", hipGetErrorString(e));
    return ok();
  });
}

}  // extern "C"
