// C entry points of the operators on device arrays (jet.h): arguments are
// checked, the GPU that holds the data is made current for the launch, and the
// work is enqueued on the caller's stream.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <exception>
#include <string>

#include "kernels.h"
#include "op_checks.h"

using namespace jet;

namespace {

// The GPU that holds p is current while this lives (the caller's one before
// and after).
struct OnDeviceOf {
  int before = -1, device = -1;
  Status st;
  OnDeviceOf(const void *p, hipStream_t stream) {
    hipPointerAttribute_t a;
    if (hipPointerGetAttributes(&a, p) != hipSuccess || a.type != hipMemoryTypeDevice) {
      (void)hipGetLastError();
      st = Status::err(JET_E_INVALID, "the arrays must be device memory");
      return;
    }
    device = a.device;
    if (stream) {
      hipDevice_t d;
      if (hipStreamGetDevice(stream, &d) != hipSuccess) {
        (void)hipGetLastError();
        st = Status::err(JET_E_DEVICE, "the stream has no device");
        return;
      }
      if ((int)d != device) {
        st = Status::err(JET_E_INVALID, "the stream belongs to another GPU than the arrays");
        return;
      }
    }
    if (hipGetDevice(&before) != hipSuccess || (before != device && hipSetDevice(device) != hipSuccess)) {
      (void)hipGetLastError();
      before = -1;
      st = Status::err(JET_E_DEVICE, "hipSetDevice failed");
    }
  }
  ~OnDeviceOf() {
    if (before >= 0 && before != device) (void)hipSetDevice(before);
  }
};

Status launched(hipError_t e, const char *what) {
  if (e == hipSuccess) return Status::ok();
  (void)hipGetLastError();
  return Status::err(JET_E_DEVICE, std::string(what) + ": " + hipGetErrorString(e));
}

jetk::QCache cache_of(const jet_qcache &c) {
  const int lb = c.block == 16 ? 4 : c.block == 32 ? 5 : c.block == 64 ? 6 : 7;
  return {c.format, lb, c.n_heads, c.head_dim, c.n_slots, (uint8_t *)c.k, (uint8_t *)c.v, c.k_exp, c.v_exp};
}
// (no sequence has more rows than the call, or more tokens than the cache)
jetk::QBatch batch_of(const jet_qcache_batch &b, const jet_qcache &c) {
  return {b.n_seq, b.n_rows, std::min(b.max_rows, b.n_rows), std::min(b.max_len, c.n_slots), b.slot0, b.len, b.row_offsets};
}
jetk::QRows rows_of(const jet_rows &r) { return {r.p, r.type, rows_aligned(r) ? 1 : 0, r.row_stride, r.head_stride}; }

constexpr int kAnyType = 1 << JET_T_F32 | 1 << JET_T_F16 | 1 << JET_T_BF16;

#define TRY(x)            \
  do {                    \
    Status s_ = (x);      \
    if (!s_) return s_;   \
  } while (0)

// Rows that are written: elements of two (row, head)s must not coincide.
Status check_out_rows(const jet_rows *r, const char *what, int types, int64_t rows, int64_t heads) {
  TRY(check_rows(r, what, types, rows));
  if ((rows > 1 && r->row_stride == 0) || (heads > 1 && r->head_stride == 0))
    return Status::err(JET_E_INVALID, std::string(what) + ": rows that are written need strides");
  return Status::ok();
}

Status move_rows(bool write, const jet_qcache *c, const jet_qcache_batch *b, const jet_rows *k, const jet_rows *v,
                 hipStream_t st) {
  TRY(check_qcache(c));
  TRY(check_batch(b));
  if (write) {
    TRY(check_rows(k, "k", kAnyType, b->n_rows));
    TRY(check_rows(v, "v", kAnyType, b->n_rows));
  } else {
    TRY(check_out_rows(k, "k", kAnyType, b->n_rows, c->n_heads));
    TRY(check_out_rows(v, "v", kAnyType, b->n_rows, c->n_heads));
  }
  if (k->type != v->type) return Status::err(JET_E_INVALID, "k and v have different types");
  if (b->n_seq == 0 || b->n_rows == 0 || c->n_slots == 0) return Status::ok();
  OnDeviceOf dev(c->k, st);
  TRY(dev.st);
  if (write) return launched(jetk::launch_qcache_write(cache_of(*c), batch_of(*b, *c), rows_of(*k), rows_of(*v), st),
                             "jet_qcache_write");
  return launched(jetk::launch_qcache_read(cache_of(*c), batch_of(*b, *c), rows_of(*k), rows_of(*v), st),
                  "jet_qcache_read");
}

Status attention(const jet_qcache *c, const jet_qcache_batch *b, int32_t n_q_heads, float scale, int32_t causal,
                 const jet_rows *q, const jet_rows *out, float *lse, void *ws, int64_t ws_bytes, hipStream_t st) {
  TRY(check_qcache(c));
  TRY(check_batch(b));
  TRY(check_q_heads(c, n_q_heads, scale));
  if (causal != 0 && causal != 1) return Status::err(JET_E_INVALID, "causal must be 0 or 1");
  TRY(check_rows(q, "q", 1 << JET_T_F16 | 1 << JET_T_BF16, b->n_rows));
  TRY(check_out_rows(out, "out", 1 << JET_T_F32 | 1 << q->type, b->n_rows, n_q_heads));
  if ((int64_t)b->n_rows * (n_q_heads / c->n_heads) > (1 << 30))
    return Status::err(JET_E_INVALID, "n_rows times the query heads of a KV head exceeds 2^30");
  if ((uintptr_t)lse % 4) return Status::err(JET_E_INVALID, "lse is not aligned");
  const jetk::QCache qc = cache_of(*c);
  const jetk::QBatch qb = batch_of(*b, *c);
  const int64_t need = jetk::qattn_workspace(qc, qb, n_q_heads);
  if (need > 0 && (!ws || ws_bytes < need || (uintptr_t)ws % 16))
    return Status::err(JET_E_INVALID, "workspace: " + std::to_string(need) + " bytes needed, 16-byte aligned");
  if (b->n_seq == 0 || b->n_rows == 0) return Status::ok();
  OnDeviceOf dev(out->p, st);
  TRY(dev.st);
  return launched(jetk::launch_qattn({qc, qb, rows_of(*q), rows_of(*out), n_q_heads, causal, scale, lse, ws}, st),
                  "jet_qcache_attention");
}

Status logits(const jet_logits_args *a, hipStream_t st) {
  TRY(check_logits(a));
  if (a->n_rows == 0) return Status::ok();
  OnDeviceOf dev(a->out, st);
  TRY(dev.st);
  const jetk::LogitsArgs l{a->n_rows,     a->vocab,       a->type,         a->n_masks,   a->logits,       a->out,
                           a->row_stride, a->out_stride,  a->hist_offsets, a->hist_ids,  a->hist_prompt,  (int)a->n_hist, nullptr,
                           a->repetition, a->presence,    a->frequency,    a->bias_offsets, a->bias_ids,  a->bias_values,
                           (int)a->n_bias, a->masks,      a->mask_stride,  a->mask_index};
  return launched(jetk::launch_logits_adjust(l, st), "jet_logits_adjust");
}

// Runs f, records a failure's message and keeps C++ exceptions inside.
template <typename F> int entry(F f) {
  try {
    clear_error();
    const Status s = f();
    return s ? JET_OK : fail(s);
  } catch (const std::exception &) {  // out of host memory
    return JET_E_OOM;
  }
}

}  // namespace

extern "C" int jet_qcache_write(const jet_qcache *cache, const jet_qcache_batch *batch, const jet_rows *k,
                                const jet_rows *v, void *hip_stream) {
  return entry([&] { return move_rows(true, cache, batch, k, v, (hipStream_t)hip_stream); });
}

extern "C" int jet_qcache_read(const jet_qcache *cache, const jet_qcache_batch *batch, const jet_rows *k,
                               const jet_rows *v, void *hip_stream) {
  return entry([&] { return move_rows(false, cache, batch, k, v, (hipStream_t)hip_stream); });
}

extern "C" int jet_qcache_attention_workspace(const jet_qcache *cache, const jet_qcache_batch *batch,
                                              int32_t n_q_heads, int64_t *out_bytes) {
  return entry([&]() -> Status {
    if (!out_bytes) return Status::err(JET_E_INVALID, "out_bytes is NULL");
    TRY(check_qcache(cache));
    TRY(check_batch_counts(batch));
    TRY(check_q_heads(cache, n_q_heads, 1.0f));
    *out_bytes = jetk::qattn_workspace(cache_of(*cache), batch_of(*batch, *cache), n_q_heads);
    return Status::ok();
  });
}

extern "C" int jet_qcache_attention(const jet_qcache *cache, const jet_qcache_batch *batch, int32_t n_q_heads,
                                    float scale, int32_t causal, const jet_rows *q, const jet_rows *out, float *lse,
                                    void *workspace, int64_t workspace_bytes, void *hip_stream) {
  return entry([&] {
    return attention(cache, batch, n_q_heads, scale, causal, q, out, lse, workspace, workspace_bytes,
                     (hipStream_t)hip_stream);
  });
}

extern "C" int jet_logits_adjust(const jet_logits_args *args, void *hip_stream) {
  return entry([&] { return logits(args, (hipStream_t)hip_stream); });
}
