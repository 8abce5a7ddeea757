// Host-side checks of the operators on device arrays (jet.h). No GPU is
// touched: what can be refused is refused before anything is enqueued.
#pragma once

#include "host.h"

namespace jet {

Status check_qcache(const jet_qcache *c);
Status check_batch_counts(const jet_qcache_batch *b);  // without the device arrays
Status check_batch(const jet_qcache_batch *b);
// types: a set of allowed 1 << JET_T_*; rows: how many the call has
Status check_rows(const jet_rows *r, const char *what, int types, int64_t rows);
// Whether rows of r can be moved in 16-byte vectors.
bool rows_aligned(const jet_rows &r);
Status check_q_heads(const jet_qcache *c, int32_t n_q_heads, float scale);
Status check_logits(const jet_logits_args *a);
// Rules of a trace of n_steps tokens for each of n_q questions. Contexts and
// traces lie in rows of one length, of kMaxTraceTokens in all at most.
constexpr int64_t kMaxTraceTokens = (int64_t)1 << 30;
Status check_rules(const jet_trace_rules *r, int32_t n_q, int32_t n_steps, int64_t vocab);
inline int type_bytes(int type) { return type == JET_T_F32 ? 4 : 2; }

}  // namespace jet
