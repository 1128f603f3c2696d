// Host-side validation of the C ABI (plain C++: built into libnovakv and, by
// the tests, into a sanitizer-checked host program).
#include "host_checks.h"

#include <stdarg.h>
#include <stdio.h>
#include <stdlib.h>

#include <atomic>
#include <string>
#include <unordered_map>
#include <unordered_set>
#include <vector>

namespace novakv {
namespace host {

thread_local std::string g_last_error;

nova_kv_status fail(nova_kv_status s, const char *fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  g_last_error = buf;
  return s;
}

nova_kv_status ok() {
  g_last_error.clear();
  return NOVA_KV_OK;
}

bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// Tag of the split exchange of the next decode call: every call gets a new
// nonzero number (the workspace's words of one call are never taken for
// another's; zero marks a never-written word).  A captured call's replays
// all carry its epoch and empty what they exchange; its epoch is even, so no
// directly launched call (odd epochs, whose words stay) ever shares it.
uint32_t next_epoch(bool captured) {
  static std::atomic<uint32_t> counter{0};
  uint32_t e;
  do {
    const uint32_t c = counter.fetch_add(1, std::memory_order_relaxed);
    e = captured ? (c + 1) << 1 : (c << 1) | 1u;
  } while (e == 0);
  return e;
}

static thread_local int g_new_token_polls = -1;
int new_token_polls() { return g_new_token_polls >= 0 ? g_new_token_polls : 512; }

nova_kv_status check_params(const nova_kv_params *p, bool need_encode, bool need_decode) {
  if (!p) return fail(NOVA_KV_ERR_INVALID_ARG, "params is NULL");
  if (p->num_kv_heads <= 0) return fail(NOVA_KV_ERR_INVALID_ARG, "num_kv_heads must be > 0");
  if (p->group_dim <= 0 || p->head_dim <= 0 || p->head_dim % p->group_dim != 0)
    return fail(NOVA_KV_ERR_INVALID_ARG, "head_dim (%d) must be a positive multiple of group_dim (%d)",
                p->head_dim, p->group_dim);
  if (p->codebook_size <= 0) return fail(NOVA_KV_ERR_INVALID_ARG, "codebook_size must be > 0");
  if (p->group_dim != novakv::kGroupDim)
    return fail(NOVA_KV_ERR_UNSUPPORTED, "group_dim %d unsupported (only 4)", p->group_dim);
  if (p->codebook_size != novakv::kCodebookSize)
    return fail(NOVA_KV_ERR_UNSUPPORTED, "codebook_size %d unsupported (only 256)", p->codebook_size);
  if (p->head_dim != 64 && p->head_dim != 128)
    return fail(NOVA_KV_ERR_UNSUPPORTED, "head_dim %d unsupported (64 or 128)", p->head_dim);
  if ((p->flags & ~(NOVA_KV_KEY_SCALE | NOVA_KV_FP8_CODEBOOKS | NOVA_KV_SQ_VALUES | NOVA_KV_BF16_TRANSFORMS)) != 0)
    return fail(NOVA_KV_ERR_UNSUPPORTED,
                "flags 0x%x unsupported (NOVA_KV_KEY_SCALE, NOVA_KV_FP8_CODEBOOKS, NOVA_KV_SQ_VALUES, "
                "NOVA_KV_BF16_TRANSFORMS)", p->flags);
  const bool sq = (p->flags & NOVA_KV_SQ_VALUES) != 0;  // cb_v unused
  if (!p->kbar || !p->cb_k || (!sq && !p->cb_v)) return fail(NOVA_KV_ERR_INVALID_ARG, "kbar/cb_k/cb_v is NULL");
  if (!aligned(p->cb_k, 16) || (!sq && !aligned(p->cb_v, 16)))
    return fail(NOVA_KV_ERR_INVALID_ARG, "codebooks must be 16-byte aligned");
  if (need_encode && (!p->t_k || !p->t_v)) return fail(NOVA_KV_ERR_INVALID_ARG, "t_k/t_v is NULL");
  if (need_decode && (!p->t_k_inv_t || !p->t_v))
    return fail(NOVA_KV_ERR_INVALID_ARG, "t_k_inv_t/t_v is NULL");
  if (!aligned(p->kbar, 16) || !aligned(p->t_v, 16) || (need_encode && !aligned(p->t_k, 16)) ||
      (need_decode && !aligned(p->t_k_inv_t, 16)))
    return fail(NOVA_KV_ERR_INVALID_ARG, "kbar and transforms must be 16-byte aligned");
  return NOVA_KV_OK;
}

nova_kv_status check_layout(const nova_kv_layout *lay) {
  if (!lay) return fail(NOVA_KV_ERR_INVALID_ARG, "layout is NULL");
  if (lay->block_size <= 0 || lay->blocks_per_seq <= 0)
    return fail(NOVA_KV_ERR_INVALID_ARG, "block_size and blocks_per_seq must be > 0");
  if (static_cast<long long>(lay->block_size) * lay->blocks_per_seq > (1LL << 30))
    return fail(NOVA_KV_ERR_INVALID_ARG, "per-sequence capacity too large");
  return NOVA_KV_OK;
}

// The scale pool of the key-scale format (ignored otherwise).
nova_kv_status check_scales(const nova_kv_params *p, const void *k_scales) {
  if (!(p->flags & NOVA_KV_KEY_SCALE)) return NOVA_KV_OK;
  if (!k_scales) return fail(NOVA_KV_ERR_INVALID_ARG, "k_scales is NULL in the key-scale format");
  if (!aligned(k_scales, 2)) return fail(NOVA_KV_ERR_INVALID_ARG, "k_scales must be 2-byte aligned");
  return NOVA_KV_OK;
}

// The sink-plus-recent band (NULL: none).
nova_kv_status check_band(const nova_kv_band *band) {
  if (!band) return NOVA_KV_OK;
  if (band->n_sink < 0 || band->n_rec < 0) return fail(NOVA_KV_ERR_INVALID_ARG, "band sizes must be >= 0");
  const long long nb = static_cast<long long>(band->n_sink) + band->n_rec;
  if (nb < 1 || nb > NOVA_KV_MAX_BAND)
    return fail(NOVA_KV_ERR_INVALID_ARG, "band of %lld positions (1 .. %d)", nb, NOVA_KV_MAX_BAND);
  if (!band->k || !band->v) return fail(NOVA_KV_ERR_INVALID_ARG, "band k or v is NULL");
  if (!aligned(band->k, 16) || !aligned(band->v, 16))
    return fail(NOVA_KV_ERR_INVALID_ARG, "band buffers must be 16-byte aligned");
  return NOVA_KV_OK;
}

// The (scale, offset) pool of the scalar value arm (ignored otherwise).
nova_kv_status check_sq(const nova_kv_params *p, const void *v_sq) {
  if (!(p->flags & NOVA_KV_SQ_VALUES)) return NOVA_KV_OK;
  if (!v_sq) return fail(NOVA_KV_ERR_INVALID_ARG, "v_sq is NULL in the scalar value format");
  if (!aligned(v_sq, 4)) return fail(NOVA_KV_ERR_INVALID_ARG, "v_sq must be 4-byte aligned");
  return NOVA_KV_OK;
}

nova_kv_status check_rotary(const nova_kv_rotary *r, bool with_q, bool with_k) {
  if (!r) return fail(NOVA_KV_ERR_INVALID_ARG, "rotary is NULL");
  if (r->num_kv_heads <= 0 || r->num_q_heads <= 0 || r->num_q_heads % r->num_kv_heads != 0)
    return fail(NOVA_KV_ERR_INVALID_ARG, "num_q_heads (%d) must be a positive multiple of num_kv_heads (%d)",
                r->num_q_heads, r->num_kv_heads);
  if (r->num_q_heads > (1 << 16)) return fail(NOVA_KV_ERR_UNSUPPORTED, "num_q_heads > 65536");
  if (r->head_dim != 64 && r->head_dim != 128)
    return fail(NOVA_KV_ERR_UNSUPPORTED, "head_dim %d unsupported (64 or 128)", r->head_dim);
  if (r->rotary_dim < 0 || r->rotary_dim > r->head_dim)
    return fail(NOVA_KV_ERR_INVALID_ARG, "rotary_dim %d outside [0, %d]", r->rotary_dim, r->head_dim);
  if (r->rotary_dim % 8 != 0)
    return fail(NOVA_KV_ERR_UNSUPPORTED, "rotary_dim %d unsupported (a multiple of 8)", r->rotary_dim);
  if (r->interleaved != 0 && r->interleaved != 1)
    return fail(NOVA_KV_ERR_INVALID_ARG, "interleaved must be 0 or 1");
  if (r->rotary_dim > 0) {
    if (!r->cos_sin || r->num_positions <= 0)
      return fail(NOVA_KV_ERR_INVALID_ARG, "cos_sin is NULL or num_positions not > 0");
    if (!aligned(r->cos_sin, 16)) return fail(NOVA_KV_ERR_INVALID_ARG, "cos_sin must be 16-byte aligned");
  }
  if ((with_q && r->q_norm && !aligned(r->q_norm, 16)) || (with_k && r->k_norm && !aligned(r->k_norm, 16)))
    return fail(NOVA_KV_ERR_INVALID_ARG, "norm weights must be 16-byte aligned");
  if ((r->q_norm_per_head & ~1) || (r->k_norm_per_head & ~1))
    return fail(NOVA_KV_ERR_INVALID_ARG, "q_norm_per_head and k_norm_per_head must be 0 or 1");
  if ((r->q_norm || r->k_norm) && !(r->eps >= 0.f)) return fail(NOVA_KV_ERR_INVALID_ARG, "eps must be >= 0");
  return NOVA_KV_OK;
}

nova_kv_status check_rows(const char *name, const nova_kv_rows *rows, const void *out, nova_kv_dtype dtype,
                          bool need_out) {
  if (!rows) {
    if (out) return fail(NOVA_KV_ERR_INVALID_ARG, "an output of %s without its rows", name);
    return NOVA_KV_OK;
  }
  if (!rows->data || (need_out && !out)) return fail(NOVA_KV_ERR_INVALID_ARG, "%s: data or output is NULL", name);
  if (!aligned(rows->data, dtype == NOVA_KV_BF16 ? 2 : 4))
    return fail(NOVA_KV_ERR_INVALID_ARG, "%s: data must be aligned to its elements", name);
  if (out && !aligned(out, 16)) return fail(NOVA_KV_ERR_INVALID_ARG, "%s: the output must be 16-byte aligned", name);
  if (rows->batch_stride < 0 || rows->token_stride < 0 || rows->batch_stride > (1LL << 40) ||
      rows->token_stride > (1LL << 40))
    return fail(NOVA_KV_ERR_INVALID_ARG, "%s: strides outside [0, 2^40]", name);
  return NOVA_KV_OK;
}

nova_kv_status check_overlaps(const nova_kv_rotary *r, const nova_kv_rows *q, const nova_kv_rows *k,
                              const nova_kv_rows *v, nova_kv_dtype dtype, int32_t batch, int32_t n_new,
                              const void *q_out, const void *k_out, const void *v_out) {
  const char *names[3] = {"q", "k", "v"};
  const nova_kv_rows *rows[3] = {q, k, v};
  const void *outs[3] = {q_out, k_out, v_out};
  // the addresses [lo, hi) of each input and output, in 128 bits (strides reach 2^40 elements)
  typedef unsigned __int128 wide;
  wide in_lo[3] = {}, in_hi[3] = {}, out_lo[3] = {}, out_hi[3] = {};
  bool dense[3] = {};
  const int elem = dtype == NOVA_KV_BF16 ? 2 : 4;
  for (int i = 0; i < 3; ++i) {
    const long long width = static_cast<long long>(i == 0 ? r->num_q_heads : r->num_kv_heads) * r->head_dim;
    if (rows[i]) {
      in_lo[i] = reinterpret_cast<uintptr_t>(rows[i]->data);
      in_hi[i] = in_lo[i] + (static_cast<wide>(batch - 1) * rows[i]->batch_stride +
                             static_cast<wide>(n_new - 1) * rows[i]->token_stride + width) * elem;
      dense[i] = (n_new == 1 || rows[i]->token_stride == width) && (batch == 1 || rows[i]->batch_stride == n_new * width);
    }
    if (outs[i]) {
      out_lo[i] = reinterpret_cast<uintptr_t>(outs[i]);
      out_hi[i] = out_lo[i] + static_cast<wide>(batch) * n_new * width * elem;
    }
  }
  for (int o = 0; o < 3; ++o) {
    for (int i = 0; i < 3; ++i) {
      if (i != o && out_lo[o] < out_hi[i] && out_lo[i] < out_hi[o])
        return fail(NOVA_KV_ERR_INVALID_ARG, "the outputs of %s and %s overlap", names[o], names[i]);
      if (out_lo[o] < in_hi[i] && in_lo[i] < out_hi[o] && !(i == o && dense[i] && in_lo[i] == out_lo[o]))
        return fail(NOVA_KV_ERR_INVALID_ARG, "the output of %s overlaps the rows of %s", names[o], names[i]);
    }
  }
  return NOVA_KV_OK;
}

nova_kv_status check_axes(const nova_kv_axes *axes, const nova_kv_rotary *r, const int32_t *positions) {
  if (!axes) return fail(NOVA_KV_ERR_INVALID_ARG, "axes is NULL");
  if (axes->num_axes < 1 || axes->num_axes > NOVA_KV_MAX_AXES)
    return fail(NOVA_KV_ERR_INVALID_ARG, "%d axes (1 .. %d)", axes->num_axes, NOVA_KV_MAX_AXES);
  if (r->rotary_dim == 0) return fail(NOVA_KV_ERR_INVALID_ARG, "positions of several axes need a rotation");
  for (int j = 0; j < r->rotary_dim / 2; ++j)
    if (axes->pair_axis[j] >= axes->num_axes)
      return fail(NOVA_KV_ERR_INVALID_ARG, "pair %d follows axis %d of %d", j, axes->pair_axis[j], axes->num_axes);
  if (!positions) return fail(NOVA_KV_ERR_INVALID_ARG, "positions is NULL");
  return NOVA_KV_OK;
}

nova_kv_status check_read_outputs(nova_kv_dtype dtype, int32_t batch, int32_t n, int32_t heads, int32_t head_dim,
                                  const void *k_out, const void *v_out) {
  if (dtype != NOVA_KV_F32 && dtype != NOVA_KV_BF16)
    return fail(NOVA_KV_ERR_INVALID_ARG, "dtype must be NOVA_KV_F32 or NOVA_KV_BF16");
  if (batch < 0 || n < 0) return fail(NOVA_KV_ERR_INVALID_ARG, "batch and n must be >= 0");
  if (batch > 65535) return fail(NOVA_KV_ERR_INVALID_ARG, "batch > 65535");
  if (batch == 0 || n == 0) return NOVA_KV_OK;
  // a launch's threads: 512 for 64 tokens of a head and side
  if ((static_cast<long long>(n) + 63) / 64 * batch > (1LL << 21) / heads)
    return fail(NOVA_KV_ERR_UNSUPPORTED, "too many tokens in a call");
  if (!aligned(k_out, 16) || !aligned(v_out, 16)) return fail(NOVA_KV_ERR_INVALID_ARG, "k_out and v_out must be 16-byte aligned");
  const unsigned long long bytes = static_cast<unsigned long long>(batch) * n * heads * head_dim * (dtype == NOVA_KV_BF16 ? 2 : 4);
  const unsigned long long k = reinterpret_cast<uintptr_t>(k_out), v = reinterpret_cast<uintptr_t>(v_out);
  if (k_out && v_out && (k < v ? v - k : k - v) < bytes) return fail(NOVA_KV_ERR_INVALID_ARG, "k_out and v_out overlap");
  return NOVA_KV_OK;
}

nova_kv_status check_q4_cache(const nova_kv_q4_cache *c) {
  if (!c) return fail(NOVA_KV_ERR_INVALID_ARG, "cache is NULL");
  if (c->num_kv_heads <= 0) return fail(NOVA_KV_ERR_INVALID_ARG, "num_kv_heads must be > 0");
  if (c->head_dim != 64 && c->head_dim != 128)
    return fail(NOVA_KV_ERR_UNSUPPORTED, "head_dim %d unsupported (64 or 128)", c->head_dim);
  const nova_kv_status st = check_layout(&c->layout);
  if (st != NOVA_KV_OK) return st;
  if (c->num_blocks <= 0) return fail(NOVA_KV_ERR_INVALID_ARG, "num_blocks must be > 0");
  const long long rows = static_cast<long long>(c->num_blocks) * c->layout.block_size;  // < 2^61
  if (rows > 0xffffffffLL / c->num_kv_heads)
    return fail(NOVA_KV_ERR_UNSUPPORTED, "a pool of more than 2^32 - 1 rows");
  if (!c->k_codes || !c->v_codes || !c->k_sq || !c->v_sq) return fail(NOVA_KV_ERR_INVALID_ARG, "a cache pool is NULL");
  if (!aligned(c->k_codes, 16) || !aligned(c->v_codes, 16))
    return fail(NOVA_KV_ERR_INVALID_ARG, "code pools must be 16-byte aligned");
  if (!aligned(c->k_sq, 4) || !aligned(c->v_sq, 4))
    return fail(NOVA_KV_ERR_INVALID_ARG, "k_sq and v_sq must be 4-byte aligned");
  return NOVA_KV_OK;
}

namespace {

long long capacity_of(const nova_kv_layout *lay) {
  return static_cast<long long>(lay->block_size) * lay->blocks_per_seq;
}

}  // namespace

nova_kv_status check_metadata(const nova_kv_layout *lay, int32_t num_blocks, int32_t batch,
                              const int32_t *seq_lens, int32_t max_seq_len, const int32_t *start_pos,
                              int32_t n_new, const int32_t *new_lens, bool may_be_absent) {
  nova_kv_status st = check_layout(lay);
  if (st != NOVA_KV_OK) return st;
  if (batch < 0 || n_new < 0) return fail(NOVA_KV_ERR_INVALID_ARG, "batch and n_new must be >= 0");
  const long long cap = capacity_of(lay);
  if (seq_lens && (max_seq_len < 0 || max_seq_len > cap))
    return fail(NOVA_KV_ERR_INVALID_ARG, "max_seq_len %d outside [0, %lld]", max_seq_len, cap);
  const bool step_write = !start_pos && seq_lens && n_new == 1;
  if (!start_pos && !step_write && n_new > 0)
    return fail(NOVA_KV_ERR_INVALID_ARG, "writes need start_pos (or seq_lens with n_new == 1)");
  const int bs = lay->block_size, bps = lay->blocks_per_seq;
  // physical block of logical block blk of sequence b (-1: absent), or a failure
  auto phys_of = [&](int b, long long blk, long long *phys) -> nova_kv_status {
    if (blk < 0 || blk >= bps)
      return fail(NOVA_KV_ERR_INVALID_ARG, "sequence %d: block %lld outside [0, %d)", b, blk, bps);
    const long long logical = static_cast<long long>(b) * bps + blk;
    const long long p = lay->block_table ? lay->block_table[logical] : logical;
    *phys = -1;
    if (may_be_absent && p < 0) return NOVA_KV_OK;
    if (p < 0 || (num_blocks > 0 && p >= num_blocks))
      return fail(NOVA_KV_ERR_INVALID_ARG, "sequence %d: block %lld maps to physical block %lld outside [0, %d)", b,
                  blk, p, num_blocks > 0 ? num_blocks : 0x7fffffff);
    *phys = p;
    return NOVA_KV_OK;
  };
  if (seq_lens) {
    for (int b = 0; b < batch; ++b)
      if (seq_lens[b] < 0 || seq_lens[b] > max_seq_len)
        return fail(NOVA_KV_ERR_INVALID_ARG, "seq_lens[%d] = %d outside [0, max_seq_len = %d]", b, seq_lens[b],
                    max_seq_len);
  }
  // written rows: physical row -> sequence, and physical blocks written
  std::unordered_map<long long, int> row_writer;
  std::unordered_map<long long, int> block_writer;
  for (int b = 0; b < batch; ++b) {
    long long w0 = 0, w1 = 0;  // written positions [w0, w1)
    if (start_pos) {
      const int32_t count = !new_lens ? n_new : new_lens[b] < 0 ? 0 : new_lens[b] < n_new ? new_lens[b] : n_new;
      w0 = start_pos[b];
      w1 = w0 + count;
      if (count > 0 && (w0 < 0 || w1 > cap))
        return fail(NOVA_KV_ERR_INVALID_ARG, "sequence %d writes positions [%lld, %lld) outside [0, %lld)", b, w0,
                    w1, cap);
    } else if (step_write && seq_lens[b] > 0) {
      w0 = seq_lens[b] - 1;
      w1 = seq_lens[b];
    }
    for (long long t = w0; t < w1; ++t) {
      long long p = 0;
      if ((st = phys_of(b, t / bs, &p)) != NOVA_KV_OK) return st;
      if (p < 0) continue;
      const long long row = p * bs + t % bs;
      auto it = row_writer.emplace(row, b);
      if (!it.second)
        return fail(NOVA_KV_ERR_INVALID_ARG, "sequences %d and %d write the same row (physical block %lld, row %lld)",
                    it.first->second, b, p, t % bs);
      auto bw = block_writer.emplace(p, b);
      if (!bw.second && bw.first->second != b) bw.first->second = -1;  // written by several sequences
    }
  }
  if (seq_lens) {
    for (int b = 0; b < batch; ++b) {
      const int s = seq_lens[b];
      // every block read must map into the pool and must not be written by
      // another sequence in the same call
      const long long nblk = (static_cast<long long>(s) + bs - 1) / bs;
      for (long long blk = 0; blk < nblk; ++blk) {
        long long p = 0;
        if ((st = phys_of(b, blk, &p)) != NOVA_KV_OK) return st;
        if (p < 0) continue;
        auto it = block_writer.find(p);
        if (it != block_writer.end() && it->second != b)
          return fail(NOVA_KV_ERR_INVALID_ARG,
                      "sequence %d reads physical block %lld, which another sequence writes in the same call", b, p);
      }
    }
  }
  return ok();
}

nova_kv_status check_reads(const nova_kv_layout *lay, int32_t num_blocks, int32_t batch, const int32_t *start_pos,
                           int32_t n, const int32_t *lens, const int32_t *seq_lens, const nova_kv_band *band,
                           bool may_be_absent) {
  const long long cap = capacity_of(lay);
  for (int b = 0; b < batch; ++b) {
    if (seq_lens && (seq_lens[b] < 0 || seq_lens[b] > cap))
      return fail(NOVA_KV_ERR_INVALID_ARG, "seq_lens[%d] = %d outside [0, %lld]", b, seq_lens[b], cap);
    const long long size = seq_lens ? seq_lens[b] : cap, from = start_pos[b];
    const long long to = from + (!lens ? n : lens[b] < 0 ? 0 : lens[b] < n ? lens[b] : n);
    if (from < to && (from < 0 || to > size))
      return fail(NOVA_KV_ERR_INVALID_ARG, "sequence %d: positions [%lld, %lld) are read of [0, %lld)", b, from, to, size);
    for (long long t = from; t < to; ++t) {
      if (band && (t < band->n_sink || t >= size - band->n_rec)) continue;
      const long long blk = t / lay->block_size, logical = static_cast<long long>(b) * lay->blocks_per_seq + blk;
      const long long p = lay->block_table ? lay->block_table[logical] : logical;
      if (may_be_absent && p < 0) continue;
      if (p < 0 || (num_blocks > 0 && p >= num_blocks))
        return fail(NOVA_KV_ERR_INVALID_ARG, "sequence %d: block %lld maps to physical block %lld outside [0, %d)", b, blk,
                    p, num_blocks > 0 ? num_blocks : 0x7fffffff);
    }
  }
  return NOVA_KV_OK;
}

nova_kv_status check_attended(const nova_kv_layout *lay, int32_t num_blocks, int32_t batch, int32_t n_q,
                              const int32_t *q_lens, const int32_t *seq_lens, int32_t max_seq_len, int32_t window,
                              const nova_kv_band *band) {
  for (int b = 0; b < batch; ++b) {
    const long long size = seq_lens[b];
    if (size < 0 || size > max_seq_len)
      return fail(NOVA_KV_ERR_INVALID_ARG, "seq_lens[%d] = %d outside [0, max_seq_len = %d]", b, seq_lens[b], max_seq_len);
    const long long queries = !q_lens ? n_q : q_lens[b] < 0 ? 0 : q_lens[b] < n_q ? q_lens[b] : n_q;
    if (queries == 0) continue;
    long long from = window > 0 && size - queries + 1 > window ? size - queries + 1 - window : 0, to = size;
    if (band) {
      if (from < band->n_sink) from = band->n_sink;
      if (to > size - band->n_rec) to = size - band->n_rec;
    }
    // Kernels that look up aligned runs of 16 positions do so in blocks of a multiple of 16 rows: the same blocks.
    for (long long blk = from / lay->block_size; from < to && blk <= (to - 1) / lay->block_size; ++blk) {
      const long long logical = static_cast<long long>(b) * lay->blocks_per_seq + blk;
      const long long p = lay->block_table ? lay->block_table[logical] : logical;
      if (p < 0 || (num_blocks > 0 && p >= num_blocks))
        return fail(NOVA_KV_ERR_INVALID_ARG, "sequence %d: block %lld maps to physical block %lld outside [0, %d)", b, blk,
                    p, num_blocks > 0 ? num_blocks : 0x7fffffff);
    }
  }
  return NOVA_KV_OK;
}

namespace {

int32_t env_debug() {
  const char *e = getenv("NOVA_KV_DEBUG");
  return e && atoi(e) != 0 ? 1 : 0;
}

std::atomic<int32_t> g_debug{env_debug()};
std::atomic<int32_t> g_debug_blocks{0};

}  // namespace

bool debug_enabled() { return g_debug.load(std::memory_order_relaxed) != 0; }
int32_t debug_num_blocks() { return g_debug_blocks.load(std::memory_order_relaxed); }

}  // namespace host
}  // namespace novakv

using namespace novakv::host;

extern "C" {

const char *nova_kv_status_string(nova_kv_status s) {
  switch (s) {
    case NOVA_KV_OK: return "ok";
    case NOVA_KV_ERR_INVALID_ARG: return "invalid argument";
    case NOVA_KV_ERR_UNSUPPORTED: return "unsupported configuration";
    case NOVA_KV_ERR_WORKSPACE: return "workspace missing or too small";
    case NOVA_KV_ERR_HIP: return "HIP runtime error";
  }
  return "unknown status";
}

const char *nova_kv_last_error(void) { return g_last_error.c_str(); }

nova_kv_status nova_kv_check_metadata(const nova_kv_layout *layout, int32_t num_blocks, int32_t batch,
                                      const int32_t *seq_lens, int32_t max_seq_len, const int32_t *start_pos,
                                      int32_t n_new) {
  return check_metadata(layout, num_blocks, batch, seq_lens, max_seq_len, start_pos, n_new);
}

void nova_kv_set_debug(int32_t on, int32_t num_blocks) {
  g_debug_blocks.store(num_blocks, std::memory_order_relaxed);
  g_debug.store(on ? 1 : 0, std::memory_order_relaxed);
}

void nova_kv_test_new_token_polls(int32_t polls) { g_new_token_polls = polls; }

}  // extern "C"
