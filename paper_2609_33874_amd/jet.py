"""ctypes binding of libjet.so (the C ABI declared in include/jet.h).

Argument marshalling only: every step of the scoring path runs in the HIP
library. Functions keep the C names. Arrays may be numpy arrays (host) or
torch tensors (host or, where jet.h allows device memory, on the model's
GPU). Loading fails loudly when the library has not been built.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libjet.so")

JET_OK, JET_E_INVALID, JET_E_CAPACITY, JET_E_OOM, JET_E_DEVICE, JET_E_IO = range(6)
JET_BF16, JET_FP32, JET_BF16_SINGLE, JET_F16, JET_F16P = 0, 1, 2, 3, 4
JET_CHOICE, JET_BINARY, JET_ORDINAL = 0, 1, 2
JET_FLAG_KERNEL_TIMING = 1
JET_FLAG_RECORD_ROUTES = 2
JET_FLAG_QCACHE_INT8, JET_FLAG_QCACHE_E4M3 = 4, 8
JET_NOALLOC_SCRATCH_BYTES = 64 << 20
JET_T_F32, JET_T_F16, JET_T_BF16 = 0, 1, 2
JET_QCACHE_INT8, JET_QCACHE_E4M3 = 0, 1
KERNEL_CLASSES = ["gemm_qkv", "gemm_o", "gemm_gateup", "gemm_down", "lmhead", "attn_prefix",
                  "attn_cand", "gdn", "other"]
ERROR_NAMES = {1: "JET_E_INVALID", 2: "JET_E_CAPACITY", 3: "JET_E_OOM", 4: "JET_E_DEVICE", 5: "JET_E_IO"}

# every symbol include/jet.h declares
EXPORTS = ["jet_model_load", "jet_prefill_prefix", "jet_generate_trace", "jet_score_candidates",
           "jet_score_candidates_noalloc", "jet_decide",
           "jet_answer_classes", "jet_evaluate", "jet_candidate_layout", "jet_stats_get", "jet_stats_reset", "jet_model_info",
           "jet_routes_get", "jet_prefix_free", "jet_model_free", "jet_last_error",
           "jet_qcache_write", "jet_qcache_read", "jet_qcache_attention", "jet_qcache_attention_workspace",
           "jet_logits_adjust", "jet_generate_trace_rules"]


class JetError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{ERROR_NAMES.get(code, code)}: {msg}")
        self.code = code


class jet_load_opts(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("device", ctypes.c_int32), ("max_ctx", ctypes.c_int64),
                ("prefill_token_budget", ctypes.c_int64), ("wave_token_budget", ctypes.c_int64),
                ("max_device_bytes", ctypes.c_int64), ("hip_stream", ctypes.c_void_p),
                ("flags", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class jet_stats(ctypes.Structure):
    _fields_ = [("prefix_tokens", ctypes.c_int64), ("prefix_evals", ctypes.c_int64),
                ("cand_body_tokens", ctypes.c_int64), ("scored_tokens", ctypes.c_int64),
                ("lm_rows", ctypes.c_int64), ("prefill_waves", ctypes.c_int64),
                ("score_waves", ctypes.c_int64), ("kernel_launches", ctypes.c_int64 * 9),
                ("kernel_ms", ctypes.c_double * 9), ("kernel_flops", ctypes.c_double * 9),
                ("kernel_bytes", ctypes.c_double * 9)]


class jet_trace_rules(ctypes.Structure):
    _fields_ = [("repetition", ctypes.c_float), ("presence", ctypes.c_float), ("frequency", ctypes.c_float),
                ("n_masks", ctypes.c_int32), ("context_offsets", ctypes.c_void_p), ("context_tokens", ctypes.c_void_p),
                ("bias_offsets", ctypes.c_void_p), ("bias_tokens", ctypes.c_void_p), ("bias_values", ctypes.c_void_p),
                ("masks", ctypes.c_void_p), ("mask_index", ctypes.c_void_p)]


class jet_qcache(ctypes.Structure):
    _fields_ = [("format", ctypes.c_int32), ("block", ctypes.c_int32), ("n_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("n_slots", ctypes.c_int64), ("k", ctypes.c_void_p),
                ("v", ctypes.c_void_p), ("k_exp", ctypes.c_void_p), ("v_exp", ctypes.c_void_p)]


class jet_qcache_batch(ctypes.Structure):
    _fields_ = [("n_seq", ctypes.c_int32), ("n_rows", ctypes.c_int32), ("max_rows", ctypes.c_int32),
                ("reserved", ctypes.c_int32), ("max_len", ctypes.c_int64), ("slot0", ctypes.c_void_p),
                ("len", ctypes.c_void_p), ("row_offsets", ctypes.c_void_p)]


class jet_rows(ctypes.Structure):
    _fields_ = [("p", ctypes.c_void_p), ("type", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("row_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class jet_logits_args(ctypes.Structure):
    _fields_ = [("n_rows", ctypes.c_int32), ("vocab", ctypes.c_int32), ("type", ctypes.c_int32),
                ("n_masks", ctypes.c_int32), ("logits", ctypes.c_void_p), ("out", ctypes.c_void_p),
                ("row_stride", ctypes.c_int64), ("out_stride", ctypes.c_int64), ("hist_offsets", ctypes.c_void_p),
                ("hist_ids", ctypes.c_void_p), ("hist_prompt", ctypes.c_void_p), ("n_hist", ctypes.c_int64),
                ("repetition", ctypes.c_void_p), ("presence", ctypes.c_void_p), ("frequency", ctypes.c_void_p),
                ("bias_offsets", ctypes.c_void_p), ("bias_ids", ctypes.c_void_p), ("bias_values", ctypes.c_void_p),
                ("n_bias", ctypes.c_int64), ("masks", ctypes.c_void_p), ("mask_stride", ctypes.c_int64),
                ("mask_index", ctypes.c_void_p)]


_lib = None


def lib() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        # torch ships its own HIP runtime under the same soname
        # (libamdhip64.so.7). Loading torch first makes the process use one
        # runtime for both, so device pointers and streams can be shared; if
        # libjet came first, torch could not initialise its runtime later.
        try:
            import torch  # noqa: F401
        except ImportError:
            pass
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is not built; run `python -m paper_2609_33874_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        P, I32, I64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
        L.jet_model_load.argtypes = [ctypes.c_char_p, ctypes.POINTER(jet_load_opts), ctypes.POINTER(P)]
        L.jet_prefill_prefix.argtypes = [P, I32, P, P, ctypes.POINTER(P)]
        L.jet_generate_trace.argtypes = [P, P, I32, ctypes.c_float, ctypes.c_uint64, P]
        L.jet_generate_trace_rules.argtypes = [P, P, I32, ctypes.c_float, ctypes.c_uint64,
                                               ctypes.POINTER(jet_trace_rules), P]
        L.jet_score_candidates.argtypes = [P, P, P, P, P, P, P]
        L.jet_score_candidates_noalloc.argtypes = [P, P, P, P, P, P, P]
        L.jet_decide.argtypes = [I32, I32, P, P, P, P, P]
        L.jet_answer_classes.argtypes = [I32, P, P, P, P]
        L.jet_evaluate.argtypes = [I32, P, P, P, P, P, P, P, P]
        L.jet_candidate_layout.argtypes = [I32, P, P, P, I64, I64, P, P, P, P, P, P]
        L.jet_stats_get.argtypes = [P, ctypes.POINTER(jet_stats)]
        L.jet_stats_reset.argtypes = [P]
        L.jet_model_info.argtypes = [P, P, P, P, P, P]
        L.jet_routes_get.argtypes = [P, I32, P, P, P, P, I64]
        qc, qb, rows = ctypes.POINTER(jet_qcache), ctypes.POINTER(jet_qcache_batch), ctypes.POINTER(jet_rows)
        L.jet_qcache_write.argtypes = [qc, qb, rows, rows, P]
        L.jet_qcache_read.argtypes = [qc, qb, rows, rows, P]
        L.jet_qcache_attention.argtypes = [qc, qb, I32, ctypes.c_float, I32, rows, rows, P, P, I64, P]
        L.jet_qcache_attention_workspace.argtypes = [qc, qb, I32, ctypes.POINTER(I64)]
        L.jet_logits_adjust.argtypes = [ctypes.POINTER(jet_logits_args), P]
        L.jet_prefix_free.argtypes = [P]
        L.jet_prefix_free.restype = None
        L.jet_model_free.argtypes = [P]
        L.jet_model_free.restype = None
        L.jet_last_error.restype = ctypes.c_char_p
        for n in EXPORTS:
            if n not in ("jet_prefix_free", "jet_model_free", "jet_last_error"):
                getattr(L, n).restype = ctypes.c_int
        _lib = L
    return _lib


def jet_last_error() -> str:
    return lib().jet_last_error().decode()


def _check(code: int) -> None:
    if code != JET_OK:
        raise JetError(code, jet_last_error())


def _ptr(x, dtype):
    """(pointer, keepalive) for a numpy array or torch tensor of `dtype`."""
    if x is None:
        return None, None
    if hasattr(x, "data_ptr"):  # torch tensor, host or device
        import torch
        want = {np.int32: torch.int32, np.int64: torch.int64, np.float32: torch.float32}[dtype]
        if x.dtype != want or not x.is_contiguous():
            raise TypeError(f"tensor must be contiguous {want}")
        return ctypes.c_void_p(x.data_ptr()), x
    a = np.ascontiguousarray(x, dtype=dtype)
    return a.ctypes.data_as(ctypes.c_void_p), a


def jet_model_load(path: str, dtype: int = JET_BF16, device: int = 0, max_ctx: int = 0,
                   prefill_token_budget: int = 0, wave_token_budget: int = 0,
                   max_device_bytes: int = 0, hip_stream: int | None = None, flags: int = 0):
    o = jet_load_opts(dtype, device, max_ctx, prefill_token_budget, wave_token_budget,
                      max_device_bytes, hip_stream or None, flags, 0)
    h = ctypes.c_void_p()
    _check(lib().jet_model_load(path.encode(), ctypes.byref(o), ctypes.byref(h)))
    return h


def jet_prefill_prefix(model, prefix_offsets, prefix_tokens):
    po, k1 = _ptr(prefix_offsets, np.int64)
    pt, k2 = _ptr(prefix_tokens, np.int32)
    n_q = len(k1) - 1
    h = ctypes.c_void_p()
    _check(lib().jet_prefill_prefix(model, n_q, po, pt, ctypes.byref(h)))
    return h


def jet_generate_trace(model, prefix, n_q: int, n_steps: int, temperature: float = 0.0, seed: int = 0, out=None):
    """Extends every question of `prefix` by n_steps sampled tokens (in place).
    Returns the tokens as int32 [n_q, n_steps] (host), or writes them into
    `out` (a contiguous int32 tensor or array of n_q * n_steps, host or device)
    and returns it."""
    if out is None:
        out = np.empty((n_q, max(int(n_steps), 0)), np.int32)
    ot, keep = _ptr(out, np.int32)
    if isinstance(out, np.ndarray) and keep is not out:
        raise TypeError("out must be a contiguous int32 array")
    _check(lib().jet_generate_trace(model, prefix, int(n_steps), float(temperature),
                                    ctypes.c_uint64(seed & 0xFFFFFFFFFFFFFFFF), ot))
    return out


def jet_generate_trace_rules(model, prefix, n_q: int, n_steps: int, temperature: float = 0.0, seed: int = 0, out=None,
                             repetition: float = 1.0, presence: float = 0.0, frequency: float = 0.0, context=None,
                             bias=None, masks=None, mask_index=None):
    """jet_generate_trace with rules for its tokens. context: (offsets [n_q + 1],
    tokens) that count as seen for `repetition`; bias: (offsets [n_q + 1],
    tokens, values); masks: uint32 [n_masks, ceil(vocab / 32)], bit v % 32 of
    word v / 32 allows token v, with mask_index [n_q, n_steps], < 0 for none."""
    if out is None:
        out = np.empty((n_q, max(int(n_steps), 0)), np.int32)
    ot, keep = _ptr(out, np.int32)
    if isinstance(out, np.ndarray) and keep is not out:
        raise TypeError("out must be a contiguous int32 array")
    r = jet_trace_rules(repetition, presence, frequency, 0)
    held = []

    def host(x, dtype, size):
        a = np.ascontiguousarray(x, dtype=dtype)
        if a.size != size:
            raise ValueError(f"a rule's array has {a.size} elements instead of {size}")
        held.append(a)
        return a.ctypes.data if a.size else None

    if context is not None:
        off = np.ascontiguousarray(context[0], np.int64)
        r.context_offsets = host(off, np.int64, n_q + 1)
        r.context_tokens = host(context[1], np.int32, int(off[-1]))
    if bias is not None:
        off = np.ascontiguousarray(bias[0], np.int64)
        r.bias_offsets = host(off, np.int64, n_q + 1)
        r.bias_tokens = host(bias[1], np.int32, int(off[-1]))
        r.bias_values = host(bias[2], np.float32, int(off[-1]))
    if masks is not None:
        masks = np.ascontiguousarray(masks, np.uint32)
        words = (jet_model_info(model)["vocab"] + 31) // 32
        r.n_masks = masks.shape[0]
        r.masks = host(masks, np.uint32, r.n_masks * words)
    if mask_index is not None:
        r.mask_index = host(mask_index, np.int32, n_q * max(int(n_steps), 0))
    _check(lib().jet_generate_trace_rules(model, prefix, int(n_steps), float(temperature),
                                          ctypes.c_uint64(seed & 0xFFFFFFFFFFFFFFFF), ctypes.byref(r), ot))
    return out


def jet_score_candidates(model, prefix, q_cand_offsets, cand_tok_offsets, cand_tokens,
                         out_token_logprob=True, out_cand_sum=None, _entry="jet_score_candidates"):
    """Returns (token log-probs or None, candidate sums). Pass torch tensors as
    outputs to have the library write them in place (host or device)."""
    qo, k1 = _ptr(q_cand_offsets, np.int64)
    co, k2 = _ptr(cand_tok_offsets, np.int64)
    ct, k3 = _ptr(cand_tokens, np.int32)
    n_cand = len(k2) - 1
    n_tok = int(k2[-1])
    if out_cand_sum is None:
        out_cand_sum = np.empty(n_cand, np.float32)
    if out_token_logprob is True:
        out_token_logprob = np.empty(n_tok, np.float32)
    elif out_token_logprob is False:
        out_token_logprob = None
    ot, k4 = _ptr(out_token_logprob, np.float32) if out_token_logprob is not None else (None, None)
    os_, k5 = _ptr(out_cand_sum, np.float32)
    if isinstance(out_cand_sum, np.ndarray) and k5 is not out_cand_sum:
        raise TypeError("out_cand_sum must be a contiguous float32 array")
    if isinstance(out_token_logprob, np.ndarray) and k4 is not out_token_logprob:
        raise TypeError("out_token_logprob must be a contiguous float32 array")
    _check(getattr(lib(), _entry)(model, prefix, qo, co, ct, ot, os_))
    return out_token_logprob, out_cand_sum


def jet_score_candidates_noalloc(model, prefix, q_cand_offsets, cand_tok_offsets, cand_tokens,
                                 out_token_logprob=True, out_cand_sum=None):
    """jet_score_candidates with every work buffer in the library's fixed
    per-device scratch (no device allocation); same arguments and results."""
    return jet_score_candidates(model, prefix, q_cand_offsets, cand_tok_offsets, cand_tokens,
                                out_token_logprob, out_cand_sum, _entry="jet_score_candidates_noalloc")


def jet_decide(mode: int, q_cand_offsets, cand_sum):
    qo, k1 = _ptr(q_cand_offsets, np.int64)
    cs, k2 = _ptr(cand_sum, np.float32)
    n_q = len(k1) - 1
    q = np.empty(len(k2), np.float64)
    choice = np.empty(n_q, np.int32)
    value = np.full(n_q, np.nan)
    _check(lib().jet_decide(mode, n_q, qo, cs, q.ctypes.data_as(ctypes.c_void_p),
                            choice.ctypes.data_as(ctypes.c_void_p), value.ctypes.data_as(ctypes.c_void_p)))
    return q, choice, value


def jet_answer_classes(q_cand_offsets, cand_tok_offsets, cand_tokens):
    """Per candidate, the index within its question of the first candidate
    with the same token sequence (equivalent labels, Section 3.3)."""
    qo, k1 = _ptr(q_cand_offsets, np.int64)
    co, k2 = _ptr(cand_tok_offsets, np.int64)
    ct, k3 = _ptr(cand_tokens, np.int32)
    out = np.empty(len(k2) - 1, np.int32)
    _check(lib().jet_answer_classes(len(k1) - 1, qo, co, ct, out.ctypes.data_as(ctypes.c_void_p)))
    return out


def jet_evaluate(q_cand_offsets, cand_sum, gold, cand_class=None):
    """(correct[n_q], gold_nll[n_q], accuracy, mean_nll) against reference
    answers, equivalent labels pooled (Section 3.3; Section 5)."""
    qo, k1 = _ptr(q_cand_offsets, np.int64)
    cs, k2 = _ptr(cand_sum, np.float32)
    gd, k3 = _ptr(gold, np.int32)
    cc, k4 = (None, None) if cand_class is None else _ptr(cand_class, np.int32)
    n_q = len(k1) - 1
    correct = np.empty(n_q, np.int32)
    nll = np.empty(n_q, np.float64)
    acc, mnll = ctypes.c_double(), ctypes.c_double()
    _check(lib().jet_evaluate(n_q, qo, cs, cc, gd, correct.ctypes.data_as(ctypes.c_void_p),
                              nll.ctypes.data_as(ctypes.c_void_p), ctypes.byref(acc), ctypes.byref(mnll)))
    return correct, nll, acc.value, mnll.value


def jet_candidate_layout(prefix_offsets, q_cand_offsets, cand_tok_offsets, max_ctx: int = 0):
    po, k1 = _ptr(prefix_offsets, np.int64)
    qo, k2 = _ptr(q_cand_offsets, np.int64)
    co, k3 = _ptr(cand_tok_offsets, np.int64)
    n_q = len(k1) - 1
    n = ctypes.c_int64()
    _check(lib().jet_candidate_layout(n_q, po, qo, co, max_ctx, 0, ctypes.byref(n), None, None, None, None, None))
    R = n.value
    out = {k: np.empty(R, np.int32) for k in ("row_pos", "row_q", "row_c", "row_tok")}
    out["lm_row"] = np.empty(int(k3[-1]), np.int32)
    P = lambda a: a.ctypes.data_as(ctypes.c_void_p)
    _check(lib().jet_candidate_layout(n_q, po, qo, co, max_ctx, R, ctypes.byref(n), P(out["row_pos"]),
                                      P(out["row_q"]), P(out["row_c"]), P(out["row_tok"]), P(out["lm_row"])))
    return out


def jet_stats_get(model) -> dict:
    s = jet_stats()
    _check(lib().jet_stats_get(model, ctypes.byref(s)))
    d = {k: getattr(s, k) for k in ("prefix_tokens", "prefix_evals", "cand_body_tokens", "scored_tokens",
                                     "lm_rows", "prefill_waves", "score_waves")}
    for f in ("kernel_launches", "kernel_ms", "kernel_flops", "kernel_bytes"):
        d[f] = dict(zip(KERNEL_CLASSES, list(getattr(s, f))))
    return d


def jet_stats_reset(model) -> None:
    _check(lib().jet_stats_reset(model))


def jet_model_info(model) -> dict:
    v, nl, mc, ni = ctypes.c_int64(), ctypes.c_int64(), ctypes.c_int64(), ctypes.c_int64()
    dt = ctypes.c_int32()
    _check(lib().jet_model_info(model, ctypes.byref(v), ctypes.byref(nl), ctypes.byref(mc), ctypes.byref(dt),
                                ctypes.byref(ni)))
    return dict(vocab=v.value, n_layers=nl.value, max_ctx=mc.value, dtype=dt.value,
                f16_inexact_weights=ni.value)


def jet_routes_get(model, which: int) -> np.ndarray:
    """Experts chosen per (layer, row) by the latest prefill (0) or scoring
    (1) call: int32 [n_layers, rows, top_k], -1 where a layer routed no row."""
    rows, nl, k = ctypes.c_int64(), ctypes.c_int32(), ctypes.c_int32()
    _check(lib().jet_routes_get(model, which, ctypes.byref(rows), ctypes.byref(nl), ctypes.byref(k), None, 0))
    out = np.empty((nl.value, rows.value, k.value), np.int32)
    _check(lib().jet_routes_get(model, which, None, None, None, out.ctypes.data_as(ctypes.c_void_p), out.size))
    return out


def jet_prefix_free(prefix) -> None:
    lib().jet_prefix_free(prefix)


def jet_model_free(model) -> None:
    lib().jet_model_free(model)


# ---------------------------------------------------------------------------
# Operators on device arrays: torch tensors on one GPU. Work is enqueued on
# `stream` (a raw hipStream_t), by default torch's current stream of that GPU.
# ---------------------------------------------------------------------------

# These calls take about as long as their smallest kernels run: their checks are
# written for few and cheap steps (devices as ordinals, shapes as they are).

_torch = None  # (torch, float types -> JET_T_*, getter of a GPU's current raw stream), once imported


def _t():
    global _torch
    if _torch is None:
        import torch
        types = {torch.float32: JET_T_F32, torch.float16: JET_T_F16, torch.bfloat16: JET_T_BF16}
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        _torch = (torch, types, raw or (lambda i: torch.cuda.current_stream(i).cuda_stream))
    return _torch


def _device_array(t, name, dtype, device, shape=None):
    """Pointer of a contiguous torch tensor on GPU `device` (None stays None)."""
    if t is None:
        return None
    if t.dtype is not dtype or t.get_device() != device:
        raise TypeError(f"{name} must be {dtype} on cuda:{device}")
    if not t.is_contiguous():
        raise TypeError(f"{name} must be contiguous")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} must have shape {shape}, not {tuple(t.shape)}")
    return t.data_ptr() or None


def _type_of(t, name):
    ty = _t()[1].get(t.dtype)
    if ty is None:
        raise TypeError(f"{name} must be float32, float16 or bfloat16")
    return ty


def _rows(t, name, heads, head_dim, device):
    shape = t.shape
    if len(shape) != 3 or shape[1] != heads or shape[2] != head_dim:
        raise ValueError(f"{name} must have shape [rows, {heads}, {head_dim}], not {list(shape)}")
    if t.get_device() != device:
        raise TypeError(f"{name} must be on cuda:{device}")
    rs, hs, es = t.stride()
    if es != 1:
        raise TypeError(f"{name} must have its last dimension contiguous")
    return jet_rows(t.data_ptr() or None, _type_of(t, name), 0, rs, hs)


def _stream(stream, device):
    return _t()[2](device) if stream is None else stream


class QCache:
    """An 8-bit attention cache over four tensors that the caller keeps: k and
    v, one byte a value, [heads, slots, head_dim]; k_exp and v_exp, uint8,
    [heads, slots // block]. `QCache.empty` makes them."""

    def __init__(self, k, v, k_exp, v_exp, block: int = 32, format: int = JET_QCACHE_INT8):
        torch = _t()[0]
        if k.dim() != 3 or k.element_size() != 1:
            raise TypeError("k must hold bytes, [heads, slots, head_dim]")
        H, S, hd = k.shape
        if not k.is_cuda:
            raise TypeError("the cache must be on a GPU")
        if v.element_size() != 1 or v.device != k.device or v.shape != k.shape:
            raise TypeError("v must be like k")
        if not (k.is_contiguous() and v.is_contiguous()):
            raise TypeError("k and v must be contiguous")
        shape = (H, S // block if block > 0 else 0)
        self.device = k.get_device()  # ordinal
        self.tensors = (k, v, k_exp, v_exp)
        self.c = jet_qcache(format, block, H, hd, S, k.data_ptr() or None, v.data_ptr() or None,
                            _device_array(k_exp, "k_exp", torch.uint8, self.device, shape),
                            _device_array(v_exp, "v_exp", torch.uint8, self.device, shape))

    @classmethod
    def empty(cls, heads: int, slots: int, head_dim: int, block: int = 32, format: int = JET_QCACHE_INT8,
              device="cuda"):
        import torch
        k, v = (torch.empty((heads, slots, head_dim), dtype=torch.int8, device=device) for _ in "kv")
        ke, ve = (torch.empty((heads, slots // block), dtype=torch.uint8, device=device) for _ in "kv")
        return cls(k, v, ke, ve, block, format)


def _batch(cache, slot0, length, n_rows, row_offsets, max_rows, max_len):
    torch, dev, n = _t()[0], cache.device, slot0.shape[0]
    off = None if row_offsets is None else _device_array(row_offsets, "row_offsets", torch.int32, dev, (n + 1,))
    if max_rows is None:
        max_rows = 1 if off is None else n_rows
    return jet_qcache_batch(n, n_rows, max_rows, 0, cache.c.n_slots if max_len is None else max_len,
                            _device_array(slot0, "slot0", torch.int64, dev, (n,)),
                            _device_array(length, "length", torch.int32, dev, (n,)), off)


def _move_rows(fn, cache, slot0, length, k, v, row_offsets, max_rows, stream):
    c, dev = cache.c, cache.device
    H, hd = c.n_heads, c.head_dim
    rk, rv, n = _rows(k, "k", H, hd, dev), _rows(v, "v", H, hd, dev), k.shape[0]
    if n != v.shape[0]:
        raise ValueError("k and v have different numbers of rows")
    if max_rows is None and row_offsets is not None:
        # (kernels walk on in a longer sequence; a launch for n rows of every
        # sequence would mostly be workgroups without any)
        max_rows = min(n, 2 * n // max(slot0.shape[0], 1) + 1)
    # (structs are passed by reference: ctypes does that itself for a POINTER argument)
    _check(fn(c, _batch(cache, slot0, length, n, row_offsets, max_rows, None), rk, rv, _stream(stream, dev)))


def jet_qcache_write(cache: QCache, slot0, length, k, v, row_offsets=None, max_rows=None, stream=None) -> None:
    """Quantises rows of k and v ([rows, heads, head_dim]) into the cache: the
    last tokens of each sequence (slot0 int64, length int32, both [n_seq];
    row_offsets int32 [n_seq + 1], None: one row each). max_rows: most rows of
    a sequence, which sizes the launch (None: about twice their mean; a longer
    sequence is worked off all the same)."""
    _move_rows(lib().jet_qcache_write, cache, slot0, length, k, v, row_offsets, max_rows, stream)


def jet_qcache_read(cache: QCache, slot0, length, k, v, row_offsets=None, max_rows=None, stream=None) -> None:
    """Reads the last tokens of each sequence back into the rows of k and v
    (arguments as jet_qcache_write's)."""
    _move_rows(lib().jet_qcache_read, cache, slot0, length, k, v, row_offsets, max_rows, stream)


def jet_qcache_attention_workspace(cache: QCache, n_seq: int, n_q_heads: int, n_rows=None, max_rows: int = 1,
                                   max_len=None) -> int:
    """Bytes of workspace that jet_qcache_attention needs for such a batch."""
    b = jet_qcache_batch(n_seq, n_seq * max_rows if n_rows is None else n_rows, max_rows, 0,
                         cache.c.n_slots if max_len is None else max_len, None, None, None)
    n = ctypes.c_int64()
    _check(lib().jet_qcache_attention_workspace(ctypes.byref(cache.c), ctypes.byref(b), n_q_heads, ctypes.byref(n)))
    return n.value


def jet_qcache_attention(cache: QCache, slot0, length, q, out, row_offsets=None, max_rows=None, max_len=None,
                         causal: bool = True, scale=None, lse=None, workspace=None, stream=None):
    """Attention of q ([rows, n_q_heads, head_dim], float16 or bfloat16) over the
    cache into `out` (q's type or float32), the rows being the last tokens of
    each sequence; lse: float32 [rows, n_q_heads] or None. scale: 1 /
    sqrt(head_dim) by default. max_rows, max_len: most rows and tokens of one
    sequence, by which the kernel and its launch are chosen (None: all rows, one
    where there are no row_offsets, and all slots: right, but slower where the
    sequences are many or much shorter than that). workspace: a uint8 tensor of
    at least jet_qcache_attention_workspace bytes for the same bounds (None: one
    is allocated, for the stream that the work runs on). Returns out."""
    c, dev, L, torch = cache.c, cache.device, lib(), _t()[0]
    hd, shape = c.head_dim, q.shape
    if len(shape) != 3 or out.shape != shape:
        raise ValueError("q and out must have shape [rows, n_q_heads, head_dim]")
    R, Hq = shape[0], shape[1]
    rq, ro = _rows(q, "q", Hq, hd, dev), _rows(out, "out", Hq, hd, dev)
    b = _batch(cache, slot0, length, R, row_offsets, max_rows, max_len)
    st = _stream(stream, dev)
    if workspace is None:
        n = ctypes.c_int64()
        _check(L.jet_qcache_attention_workspace(c, b, Hq, n))
        if n.value:
            if stream is None or stream == _stream(None, dev):
                workspace = torch.empty(n.value, dtype=torch.uint8, device=f"cuda:{dev}")
            else:
                # out of that stream's pool: a block that was freed on the current
                # one may still be in use by work that is queued there
                with torch.cuda.stream(torch.cuda.ExternalStream(stream, device=dev) if stream
                                       else torch.cuda.default_stream(dev)):
                    workspace = torch.empty(n.value, dtype=torch.uint8, device=f"cuda:{dev}")
    ws, ws_n = (None, 0) if workspace is None else (_device_array(workspace, "workspace", torch.uint8, dev),
                                                    workspace.numel())
    _check(L.jet_qcache_attention(c, b, Hq, hd ** -0.5 if scale is None else scale, 1 if causal else 0, rq, ro,
                                  _device_array(lse, "lse", torch.float32, dev, (R, Hq)), ws, ws_n, st))
    return out


def jet_logits_adjust(logits, out=None, history=None, hist_prompt=None, repetition=None, presence=None,
                      frequency=None, bias=None, masks=None, mask_index=None, stream=None):
    """Penalties for repeated tokens, biases and masks on logits [rows, vocab]
    (float32, float16 or bfloat16, any row stride). out: where to write (None:
    in place). history: (offsets int32 [rows + 1], ids int32); hist_prompt:
    int32 [rows], how many of a row's ids are its prompt. repetition, presence,
    frequency: float32 [rows]. bias: (offsets int32 [rows + 1], ids int32,
    values float32). masks: int32 [n_masks, words], bit v % 32 of word v / 32
    allows token v; mask_index: int32 [rows], < 0 for none. Returns out."""
    torch = _t()[0]
    out = logits if out is None else out
    shape = logits.shape
    if len(shape) != 2 or out.shape != shape or out.dtype is not logits.dtype:
        raise ValueError("logits and out must be [rows, vocab] of one type")
    R, V = shape
    dev = logits.get_device()
    if dev < 0 or out.get_device() != dev:
        raise TypeError("logits and out must be on one GPU")
    (ld, s1), (ld_out, o1) = logits.stride(), out.stride()
    if V > 1 and (s1 != 1 or o1 != 1):
        raise TypeError("logits and out must have contiguous rows")
    if R <= 1:
        ld, ld_out = max(ld, V), max(ld_out, V)
    i32, f32 = torch.int32, torch.float32
    a = jet_logits_args(R, V, _type_of(logits, "logits"), 0, logits.data_ptr() or None, out.data_ptr() or None, ld,
                        ld_out)
    if history is not None:
        a.hist_offsets = _device_array(history[0], "history offsets", i32, dev, (R + 1,))
        a.hist_ids, a.n_hist = _device_array(history[1], "history ids", i32, dev), history[1].numel()
    a.hist_prompt = _device_array(hist_prompt, "hist_prompt", i32, dev, (R,))
    a.repetition = _device_array(repetition, "repetition", f32, dev, (R,))
    a.presence = _device_array(presence, "presence", f32, dev, (R,))
    a.frequency = _device_array(frequency, "frequency", f32, dev, (R,))
    if bias is not None:
        a.bias_offsets = _device_array(bias[0], "bias offsets", i32, dev, (R + 1,))
        a.bias_ids, a.n_bias = _device_array(bias[1], "bias ids", i32, dev), bias[1].numel()
        a.bias_values = _device_array(bias[2], "bias values", f32, dev, (a.n_bias,))
    if masks is not None:
        if masks.dim() != 2 or (R and not masks.shape[0]):
            raise ValueError("masks must be [n_masks, words], one mask at least")
        a.masks, a.n_masks = _device_array(masks, "masks", i32, dev), masks.shape[0]
        a.mask_stride = masks.shape[1]
    a.mask_index = _device_array(mask_index, "mask_index", i32, dev, (R,))
    _check(lib().jet_logits_adjust(a, _stream(stream, dev)))
    return out
