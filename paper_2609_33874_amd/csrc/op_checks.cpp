// Checks of the operators' arguments that need no GPU.
#include "op_checks.h"

#include <algorithm>
#include <cmath>

namespace jet {

static Status bad(const std::string &m) { return Status::err(JET_E_INVALID, m); }
static bool aligned(const void *p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

Status check_qcache(const jet_qcache *c) {
  if (!c) return bad("cache is NULL");
  if (c->format != JET_QCACHE_INT8 && c->format != JET_QCACHE_E4M3) return bad("unknown cache format");
  if (c->block != 16 && c->block != 32 && c->block != 64 && c->block != 128)
    return bad("a cache block holds 16, 32, 64 or 128 tokens");
  if (c->n_heads < 1 || c->n_heads > 1024) return bad("cache n_heads must be in 1 .. 1024");
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256)
    return bad("cache head_dim must be 64, 128 or 256");
  if (c->n_slots < 0 || c->n_slots % c->block) return bad("cache n_slots must be a multiple of its block");
  if (c->n_slots > ((int64_t)1 << 40)) return bad("cache n_slots is too large");
  if (c->n_slots > 0 && (!c->k || !c->v || !c->k_exp || !c->v_exp)) return bad("a cache array is NULL");
  if (!aligned(c->k, 16) || !aligned(c->v, 16)) return bad("cache k and v must be 16-byte aligned");
  return Status::ok();
}

Status check_batch_counts(const jet_qcache_batch *b) {
  if (!b) return bad("batch is NULL");
  if (b->n_seq < 0 || b->n_seq > 65535) return bad("n_seq must be in 0 .. 65535");
  if (b->n_rows < 0 || b->n_rows > (1 << 30)) return bad("n_rows must be in 0 .. 2^30");
  if (b->max_rows < 0 || b->max_len < 0) return bad("max_rows and max_len must be >= 0");
  return Status::ok();
}

Status check_batch(const jet_qcache_batch *b) {
  Status s = check_batch_counts(b);
  if (!s) return s;
  if (b->n_seq > 0 && (!b->slot0 || !b->len)) return bad("slot0 or len is NULL");
  if (!b->row_offsets && b->n_rows < b->n_seq) return bad("without row_offsets every sequence has a row: n_rows < n_seq");
  if (!aligned(b->slot0, 8) || !aligned(b->len, 4) || !aligned(b->row_offsets, 4))
    return bad("slot0, len or row_offsets is not aligned");
  return Status::ok();
}

Status check_rows(const jet_rows *r, const char *what, int types, int64_t rows) {
  if (!r) return bad(std::string(what) + " is NULL");
  if (r->type < 0 || r->type > JET_T_BF16 || !(types & (1 << r->type)))
    return bad(std::string(what) + ": element type not taken here");
  if (!r->p && rows > 0) return bad(std::string(what) + ": array is NULL");
  if (!aligned(r->p, (size_t)type_bytes(r->type))) return bad(std::string(what) + ": array is not aligned");
  if (r->row_stride < 0 || r->head_stride < 0) return bad(std::string(what) + ": negative stride");
  if (r->row_stride > ((int64_t)1 << 40) || r->head_stride > ((int64_t)1 << 40))
    return bad(std::string(what) + ": stride is too large");
  return Status::ok();
}

bool rows_aligned(const jet_rows &r) {
  const int64_t n = 16 / type_bytes(r.type);
  return aligned(r.p, 16) && r.row_stride % n == 0 && r.head_stride % n == 0;
}

Status check_q_heads(const jet_qcache *c, int32_t n_q_heads, float scale) {
  if (!std::isfinite(scale)) return bad("scale must be finite");
  if (n_q_heads < 1 || n_q_heads % c->n_heads) return bad("n_q_heads must be a multiple of the cache's heads");
  if (n_q_heads / c->n_heads > 64) return bad("at most 64 query heads a KV head");
  if (n_q_heads > 32768) return bad("at most 32768 query heads");
  return Status::ok();
}

Status check_logits(const jet_logits_args *a) {
  if (!a) return bad("args is NULL");
  if (a->n_rows < 0 || a->n_rows > (1 << 20)) return bad("n_rows must be in 0 .. 2^20");
  if (a->vocab < 1 || a->vocab > (1 << 24)) return bad("vocab must be in 1 .. 2^24");
  if (a->type < 0 || a->type > JET_T_BF16) return bad("unknown logits type");
  if (a->row_stride < a->vocab || a->out_stride < a->vocab || a->row_stride > ((int64_t)1 << 40) ||
      a->out_stride > ((int64_t)1 << 40))
    return bad("row strides must be at least vocab");
  if (a->n_rows > 0 && (!a->logits || !a->out)) return bad("logits or out is NULL");
  const size_t es = (size_t)type_bytes(a->type);
  if (!aligned(a->logits, es) || !aligned(a->out, es)) return bad("logits or out is not aligned");
  if (a->out == a->logits && a->out_stride != a->row_stride) return bad("in place, out_stride must be row_stride");
  if (a->n_hist < 0 || a->n_hist > (1 << 30)) return bad("n_hist must be in 0 .. 2^30");
  if (a->hist_offsets && a->n_hist > 0 && !a->hist_ids) return bad("hist_ids is NULL");
  if (a->n_bias < 0 || a->n_bias > (1 << 30)) return bad("n_bias must be in 0 .. 2^30");
  if (a->bias_offsets && a->n_bias > 0 && (!a->bias_ids || !a->bias_values)) return bad("bias_ids or bias_values is NULL");
  if (a->n_masks < 0) return bad("n_masks must be >= 0");
  if (a->masks) {
    if (a->mask_stride < (a->vocab + 31) / 32 || a->mask_stride > ((int64_t)1 << 40))
      return bad("mask_stride must be at least ceil(vocab / 32) words");
    if (!a->mask_index && a->n_masks < a->n_rows) return bad("without mask_index every row has a mask: n_masks < n_rows");
  } else if (a->n_masks > 0) {
    return bad("masks is NULL");
  }
  for (const void *p : {(const void *)a->hist_offsets, (const void *)a->hist_ids, (const void *)a->hist_prompt,
                        (const void *)a->repetition, (const void *)a->presence, (const void *)a->frequency,
                        (const void *)a->bias_offsets, (const void *)a->bias_ids, (const void *)a->bias_values,
                        (const void *)a->masks, (const void *)a->mask_index})
    if (!aligned(p, 4)) return bad("an array of 32-bit values is not aligned");
  return Status::ok();
}

Status check_rules(const jet_trace_rules *r, int32_t n_q, int32_t n_steps, int64_t vocab) {
  if (!r) return Status::ok();
  if (!(r->repetition > 0.0f) || !std::isfinite(r->repetition) || !std::isfinite(1.0f / r->repetition))
    return bad("repetition must be > 0 and finite, its inverse too");
  if (!std::isfinite(r->presence) || !std::isfinite(r->frequency)) return bad("presence and frequency must be finite");
  Status s;
  if (r->context_offsets) {
    s = check_offsets(r->context_offsets, n_q, 0, "context_offsets");
    if (!s) return s;
    if (r->context_offsets[n_q] > INT32_MAX) return bad("too many context tokens");
    s = check_ids_host(r->context_tokens, r->context_offsets[n_q], vocab, "context_tokens");
    if (!s) return s;
    int64_t longest = 0;  // (every question has a row of so many tokens)
    for (int32_t q = 0; q < n_q; ++q) longest = std::max(longest, r->context_offsets[q + 1] - r->context_offsets[q]);
    if (n_q * (longest + n_steps) > kMaxTraceTokens)
      return bad("n_q times the longest context and n_steps exceeds 2^30");
  }
  if (r->bias_offsets) {
    s = check_offsets(r->bias_offsets, n_q, 0, "bias_offsets");
    if (!s) return s;
    const int64_t n = r->bias_offsets[n_q];
    if (n > (1 << 30)) return bad("too many biases");
    s = check_ids_host(r->bias_tokens, n, vocab, "bias_tokens");
    if (!s) return s;
    if (n > 0 && !r->bias_values) return bad("bias_values is NULL");
    for (int64_t i = 0; i < n; ++i)
      if (!std::isfinite(r->bias_values[i])) return bad("bias " + std::to_string(i) + " is not finite");
  }
  if (r->n_masks < 0) return bad("n_masks must be >= 0");
  if (r->n_masks > 0) {
    if (!r->masks || !r->mask_index) return bad("masks or mask_index is NULL");
    const int64_t words = (vocab + 31) / 32;
    for (int32_t m = 0; m < r->n_masks; ++m) {
      uint32_t any = 0;
      for (int64_t w = 0; w < words; ++w) {
        const uint32_t x = r->masks[(int64_t)m * words + w];
        any |= w == words - 1 && vocab % 32 ? x & ((1u << (vocab % 32)) - 1) : x;
      }
      if (!any) return bad("mask " + std::to_string(m) + " allows no token");
    }
  }
  for (int64_t i = 0; r->mask_index && i < (int64_t)n_q * n_steps; ++i)
    if (r->mask_index[i] >= r->n_masks) return bad("mask_index " + std::to_string(i) + " names no mask");
  return Status::ok();
}

}  // namespace jet
