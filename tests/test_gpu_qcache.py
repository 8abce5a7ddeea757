"""GPU: retained caches in 8 bits (JET_FLAG_QCACHE_*) and rules for traces
(jet_generate_trace_rules) through prefill, scoring and decoding, against the
fp64 oracle.

Scores: the oracle runs each prefix once, its retained K and V are rounded as
the cache's format says (in 64 bits, tests/_qcache_ref.py), and every candidate
runs against that state. The library's K and V differ from the oracle's by its
mode's rounding, so some values round to the other neighbour. With d_q the
largest change that the format itself makes to a token's log-probability in the
oracle (all values off by up to half a step, uniformly: 0.29 of a step rms):
  * JET_FP32: K and V are right to about 1e-6 of a block's largest value, 1e-4
    of a step, so one value in 10^4 moves by a step: sqrt(1e-4) / 0.29 = 0.035 of
    d_q rms; 0.25 d_q leaves room for chance, plus the mode's own tolerance;
  * JET_F16: K and V are rounded to 2^-12 of a value, up to 0.03 of a step, so
    one in 30 moves: sqrt(0.03) / 0.29 = 0.6 of d_q rms, and own rounding of the
    scores: 1.5 d_q plus the mode's tolerance.
"""
import copy
import sys

import numpy as np
import pytest

import _qcache_ref as ref
import jet_synth
import oracle
from oracle import generate as og
from oracle.model import Model, final_logprobs, forward, rmsnorm
from paper_2609_33874_amd import jet as J

from test_gpu_parity import TOL

pytestmark = pytest.mark.gpu

FLAGS = {0: J.JET_FLAG_QCACHE_INT8, 1: J.JET_FLAG_QCACHE_E4M3}
SLACK = {J.JET_FP32: 0.25, J.JET_F16: 1.5}


def log(msg):
    print(msg, file=sys.__stderr__, flush=True)


class QState:
    """A question's retained K and V per attention layer, rounded as the cache rounds them."""

    def __init__(self, state, room, fmt):
        self.caches = []
        for st in state:
            if len(st) != 3:  # a delta-rule layer's state is not a cache
                self.caches.append(None)
                continue
            n, H, hd = st[0].shape
            slots = (n + room + 31) // 32 * 32
            self.caches.append([[ref.RefCache(slots, hd, 32, fmt) for _ in range(H)] for _ in "kv"])
        self.n = 0
        self.append(state)

    def append(self, state):
        """The tokens of `state` past those held, as one write."""
        for c, st in zip(self.caches, state):
            if c is not None:
                for kv in (0, 1):
                    for h, r in enumerate(c[kv]):
                        r.write(0, self.n, st[kv][self.n:, h])
                new = len(st[2])
        self.n = new

    def rounded(self, state):
        out = []
        for c, st in zip(self.caches, state):
            if c is None:
                out.append(copy.deepcopy(st))
            else:
                k, v = (np.stack([r.values(0, self.n) for r in c[kv]], axis=1) for kv in (0, 1))
                out.append((k, v, np.arange(self.n)))
        return out


def oracle_scores(model, wl, fmt):
    """Token log-probabilities with plain and with rounded prefix caches."""
    W = model.w("lm_head")
    plain, quant = np.zeros(len(wl.cand_tokens)), np.zeros(len(wl.cand_tokens))
    for q in range(wl.n_questions):
        x = wl.prefix(q).astype(np.int64)
        hid, st = forward(model, [x], want_state=True)
        rounded = QState(st[0], 0, fmt).rounded(st[0])
        for j, y in enumerate(wl.candidates(q)):
            c = int(wl.q_cand_offsets[q]) + j
            for out, state in ((plain, st[0]), (quant, rounded)):
                rows = [hid[0][-1:]]
                if len(y) > 1:
                    rows.append(forward(model, [y[:-1].astype(np.int64)], starts=[len(x)],
                                        states=[copy.deepcopy(state)])[0][0])
                out[wl.cand_tok_offsets[c]:wl.cand_tok_offsets[c + 1]] = final_logprobs(model, np.concatenate(rows), y, W)
    return plain, quant


def scores(m, wl, fn=J.jet_score_candidates):
    p = J.jet_prefill_prefix(m, wl.prefix_offsets, wl.prefix_tokens)
    try:
        return fn(m, p, wl.q_cand_offsets, wl.cand_tok_offsets, wl.cand_tokens)
    finally:
        J.jet_prefix_free(p)


@pytest.fixture(scope="module")
def reference(model_dir):
    """(oracle plain, oracle rounded) of a workload, made once."""
    made = {}

    def get(spec, wname, n, fmt):
        key = (spec, wname, n, fmt)
        if key not in made:
            path = jet_synth.ensure_model(spec, cache_dir=model_dir)
            made[key] = oracle_scores(Model(path), jet_synth.make_workload(wname, n_questions=n), fmt)
        return made[key]
    return get


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("spec,wname,dtype", [
    ("small_gqa_bf16", "small", J.JET_FP32), ("small_gqa_bf16", "small", J.JET_F16),
    ("small_hybrid_bf16", "small_hybrid", J.JET_F16), ("small_hybrid_bf16", "small_hybrid", J.JET_FP32)])
def test_scores_with_caches_in_8_bits(spec, wname, dtype, fmt, model_dir, reference):
    path = jet_synth.ensure_model(spec, cache_dir=model_dir)
    wl = jet_synth.make_workload(wname, n_questions=5)
    plain, quant = reference(spec, wname, 5, fmt)
    d_q = np.abs(quant - plain).max()
    m = J.jet_model_load(path, dtype=dtype, flags=FLAGS[fmt])
    try:
        tok, sums = scores(m, wl)
        tok2, sums2 = scores(m, wl)
        small = J.jet_model_load(path, dtype=dtype, flags=FLAGS[fmt], prefill_token_budget=300, wave_token_budget=30)
        try:
            tok3, _ = scores(small, wl)  # several waves each way
        finally:
            J.jet_model_free(small)
        tok4, sums4 = scores(m, wl, J.jet_score_candidates_noalloc)
    finally:
        J.jet_model_free(m)
    err = np.abs(tok - quant).max()
    log(f"[qcache] {spec} dtype={dtype} fmt={fmt}: max|d tok|={err:.3e}, the format's own {d_q:.3e}")
    assert d_q > 0 and err <= TOL[dtype][0] + SLACK[dtype] * d_q
    np.testing.assert_array_equal(tok, tok2)
    np.testing.assert_array_equal(sums, sums2)
    assert np.abs(tok3 - tok).max() <= 1e-5 if dtype == J.JET_FP32 else np.abs(tok3 - quant).max() <= TOL[dtype][0] + SLACK[dtype] * d_q
    if dtype == J.JET_F16:
        np.testing.assert_array_equal(tok4, tok)
    else:
        assert np.abs(tok4 - tok).max() <= 1e-5


def test_a_candidate_scores_the_same_alone(model_dir):
    """Bitwise: among its siblings, alone, and in the order turned round."""
    path = jet_synth.ensure_model("small_gqa_bf16", cache_dir=model_dir)
    wl = jet_synth.make_workload("small", n_questions=3)
    m = J.jet_model_load(path, dtype=J.JET_F16, flags=J.JET_FLAG_QCACHE_INT8)
    try:
        p = J.jet_prefill_prefix(m, wl.prefix_offsets, wl.prefix_tokens)
        tok, sums = J.jet_score_candidates(m, p, wl.q_cand_offsets, wl.cand_tok_offsets, wl.cand_tokens)
        for q in range(wl.n_questions):
            for j, y in enumerate(wl.candidates(q)):
                c = int(wl.q_cand_offsets[q]) + j
                qo = np.array([0] * (q + 1) + [1] * (wl.n_questions - q), np.int64)
                t1, s1 = J.jet_score_candidates(m, p, qo, np.array([0, len(y)], np.int64), y)
                np.testing.assert_array_equal(t1, tok[wl.cand_tok_offsets[c]:wl.cand_tok_offsets[c + 1]])
                assert s1[0] == sums[c]
        J.jet_prefix_free(p)
    finally:
        J.jet_model_free(m)


def test_many_candidates_and_long_ones(model_dir):
    """Own rows past one block of query slots, and candidates longer than a key tile, against JET_FP32."""
    path = jet_synth.ensure_model("small_gqa_bf16", cache_dir=model_dir)
    rng = np.random.default_rng(3)
    pre = [rng.integers(0, 3000, size=n).astype(np.int32) for n in (200, 31, 1)]
    cands = [[rng.integers(0, 3000, size=n).astype(np.int32) for n in lens]
             for lens in ([150, 1, 70, 9, 9, 9, 30] + [4] * 40, [65, 64, 66, 2], [5, 1])]
    wl = jet_synth.from_lists(pre, cands)
    got = {}
    for dtype in (J.JET_FP32, J.JET_F16):
        m = J.jet_model_load(path, dtype=dtype, flags=J.JET_FLAG_QCACHE_INT8)
        try:
            got[dtype] = scores(m, wl)[0]
        finally:
            J.jet_model_free(m)
    plain, quant = oracle_scores(Model(path), wl.subset([1, 2]), 0)
    d_q = np.abs(quant - plain).max()
    n = len(quant)
    for dtype in got:
        assert np.abs(got[dtype][-n:] - quant).max() <= TOL[dtype][0] + SLACK[dtype] * d_q
    err = np.abs(got[J.JET_FP32] - got[J.JET_F16]).max()
    log(f"[qcache] long candidates: f16 and f32 differ by {err:.3e}")
    assert err <= TOL[J.JET_F16][0] + 1.5 * d_q


# ---------------------------------------------------------------------------
# traces
# ---------------------------------------------------------------------------

def logits_of(model, hid):
    return (rmsnorm(hid[-1:], model.w("final_norm"), model.eps) @ model.w("lm_head").T)[0]


@pytest.mark.parametrize("dtype,fmt,tau", [(J.JET_FP32, 0, 0.0), (J.JET_F16, 0, 0.8), (J.JET_F16, 1, 0.0),
                                           (J.JET_FP32, 1, 0.8)])
def test_traces_over_caches_in_8_bits(dtype, fmt, tau, model_dir):
    """Every token of a trace is within tolerance of the best one under the oracle's logits over rounded caches
    (which grow with the trace, token by token); scores on the extended prefix follow its rounded caches."""
    path = jet_synth.ensure_model("small_gqa_bf16", cache_dir=model_dir)
    wl = jet_synth.make_workload("small", n_questions=3)
    n, seed = 6, 77
    m = J.jet_model_load(path, dtype=dtype, flags=FLAGS[fmt])
    try:
        p = J.jet_prefill_prefix(m, wl.prefix_offsets, wl.prefix_tokens)
        trace = np.concatenate([J.jet_generate_trace(m, p, 3, k, tau, seed) for k in ((n,) if tau else (4, 2))], 1)
        tok, _ = J.jet_score_candidates(m, p, wl.q_cand_offsets, wl.cand_tok_offsets, wl.cand_tokens)
        J.jet_prefix_free(p)
    finally:
        J.jet_model_free(m)
    model = Model(path)
    W = model.w("lm_head")
    t_tol, worst, worst_s, r = TOL[dtype][0], 0.0, 0.0, 0
    for q in range(3):
        x = wl.prefix(q).astype(np.int64)
        hid, st = forward(model, [x], want_state=True)
        exact, qs = st[0], QState(st[0], n, fmt)
        z, zp = logits_of(model, hid[0]), None
        d_z = 0.0
        for t in range(n):
            y = np.array([trace[q, t]], np.int64)
            keys = og.sample_keys(z, tau, seed, q, t)
            gap = keys.max() - keys[y[0]]
            allowed = 2 * (t_tol + SLACK[dtype] * d_z) / (tau if tau else 1.0)
            assert gap <= allowed, (q, t, gap, allowed)
            worst = max(worst, gap)
            # the next token: over rounded caches, and over exact ones for what rounding changes
            h2, st2 = forward(model, [y], starts=[len(x) + t], states=[qs.rounded(exact)], want_state=True)
            hp, exact_next = forward(model, [y], starts=[len(x) + t], states=[copy.deepcopy(exact)], want_state=True)
            z, zp = logits_of(model, h2[0]), logits_of(model, hp[0])
            d_z = max(d_z, np.abs(z - zp).max())
            qs.append(st2[0])
            exact = exact_next[0]
            hid = h2
        state = qs.rounded(exact)
        for j, y in enumerate(wl.candidates(q)):
            rows = [hid[0][-1:]]
            if len(y) > 1:
                rows.append(forward(model, [y[:-1].astype(np.int64)], starts=[len(x) + n],
                                    states=[copy.deepcopy(state)])[0][0])
            want = final_logprobs(model, np.concatenate(rows), y, W)
            err = np.abs(tok[r:r + len(y)] - want).max()
            worst_s = max(worst_s, err)
            # (the trace's rows saw their own key rounded, the oracle's as it was: another d_z)
            assert err <= t_tol + (SLACK[dtype] + 1.0) * d_z
            r += len(y)
    log(f"[qcache] trace dtype={dtype} fmt={fmt} tau={tau}: largest gap {worst:.3e}, scores {worst_s:.3e}, "
        f"rounding's own {d_z:.3e}")


def words_of(allow):
    V = allow.shape[1]
    pad = np.zeros((len(allow), (V + 31) // 32 * 32), bool)
    pad[:, :V] = allow
    return np.packbits(pad, axis=1, bitorder="little").view(np.uint32)


@pytest.mark.parametrize("dtype,tau,flags", [(J.JET_FP32, 0.0, 0), (J.JET_F16, 0.9, 0), (J.JET_F16, 0.0, J.JET_FLAG_QCACHE_INT8)])
def test_traces_with_rules(dtype, tau, flags, model_dir):
    """Tokens obey the masks; each is within tolerance of the best one under the rules in 64 bits."""
    path = jet_synth.ensure_model("small_gqa_bf16", cache_dir=model_dir)
    wl = jet_synth.make_workload("small", n_questions=4)
    n, seed, V = 7, 5, 3000
    rng = np.random.default_rng(9)
    allow = rng.random((3, V)) < np.array([0.01, 0.5, 0.9])[:, None]
    allow[0, 17] = True
    mi = rng.integers(-1, 3, size=(4, n)).astype(np.int32)
    ctx = [wl.prefix(q) if q != 2 else wl.prefix(q)[:0] for q in range(4)]
    co = np.concatenate([[0], np.cumsum([len(c) for c in ctx])]).astype(np.int64)
    nb = [3, 0, 40, 1]
    bo = np.concatenate([[0], np.cumsum(nb)]).astype(np.int64)
    bt, bv = rng.integers(0, V, size=sum(nb)).astype(np.int32), rng.normal(size=sum(nb)).astype(np.float32)
    rep, pres, freq = np.float32(1.4), np.float32(0.3), np.float32(0.2)
    m = J.jet_model_load(path, dtype=dtype, flags=flags)
    try:
        p = J.jet_prefill_prefix(m, wl.prefix_offsets, wl.prefix_tokens)
        tr = J.jet_generate_trace_rules(m, p, 4, n, tau, seed, repetition=float(rep), presence=float(pres),
                                        frequency=float(freq), context=(co, np.concatenate(ctx)), bias=(bo, bt, bv),
                                        masks=words_of(allow), mask_index=mi)
        tok, _ = J.jet_score_candidates(m, p, wl.q_cand_offsets, wl.cand_tok_offsets, wl.cand_tokens)
        J.jet_prefix_free(p)
        # no rules at all: the plain call, bit for bit
        outs = []
        for f in (J.jet_generate_trace, J.jet_generate_trace_rules):
            p = J.jet_prefill_prefix(m, wl.prefix_offsets, wl.prefix_tokens)
            outs.append((f(m, p, 4, n, tau, seed),
                         J.jet_score_candidates(m, p, wl.q_cand_offsets, wl.cand_tok_offsets, wl.cand_tokens)[0]))
            J.jet_prefix_free(p)
        np.testing.assert_array_equal(outs[0][0], outs[1][0])
        np.testing.assert_array_equal(outs[0][1], outs[1][1])
        assert not np.array_equal(outs[0][0], tr)
    finally:
        J.jet_model_free(m)
    assert np.all(np.isfinite(tok))
    model = Model(path)
    # a logit's tolerance, stretched by the penalty; caches in 8 bits: what they change is bounded by the test above
    z_tol = (TOL[dtype][0] if not flags else 4 * TOL[dtype][0]) * float(rep)
    for q in range(4):
        seq = [int(x) for x in wl.prefix(q)]
        for t in range(n):
            y = int(tr[q, t])
            al = allow[mi[q, t]] if mi[q, t] >= 0 else None
            assert al is None or al[y], (q, t, y)
            h = [int(x) for x in ctx[q]] + [int(x) for x in tr[q, :t]]
            z, _ = ref.adjust(og.next_logits(model, seq), h, len(ctx[q]), float(rep), float(pres), float(freq),
                              list(zip(bt[bo[q]:bo[q + 1]].tolist(), bv[bo[q]:bo[q + 1]].astype(float).tolist())), al)
            keys = og.sample_keys(z, tau, seed, q, t)
            assert keys.max() - keys[y] <= 2 * z_tol / (tau if tau else 1.0), (q, t)
            seq.append(y)


def test_refused_rules_change_nothing(model_dir):
    path = jet_synth.ensure_model("small_gqa_bf16", cache_dir=model_dir)
    wl = jet_synth.make_workload("small", n_questions=2)
    m = J.jet_model_load(path, dtype=J.JET_F16, flags=J.JET_FLAG_QCACHE_E4M3)
    one = np.ones((1, 3000), bool)
    try:
        p = J.jet_prefill_prefix(m, wl.prefix_offsets, wl.prefix_tokens)
        args = (wl.q_cand_offsets, wl.cand_tok_offsets, wl.cand_tokens)
        tok, _ = J.jet_score_candidates(m, p, *args)
        for kw in (dict(repetition=0.0), dict(repetition=-1.0), dict(repetition=float("nan")),
                   dict(repetition=1e-45), dict(presence=float("inf")), dict(frequency=float("nan")),
                   dict(context=([0, 1, 2], [5, 3000])), dict(context=([0, 2, 1], [5])),
                   dict(bias=([0, 1, 1], [-1], [1.0])), dict(bias=([0, 1, 1], [1], [float("inf")])),
                   dict(masks=words_of(~one), mask_index=np.zeros((2, 3), np.int32)),
                   dict(masks=words_of(one), mask_index=np.ones((2, 3), np.int32)), dict(masks=words_of(one))):
            with pytest.raises(J.JetError) as e:
                J.jet_generate_trace_rules(m, p, 2, 3, **kw)
            assert e.value.code == J.JET_E_INVALID, kw
        np.testing.assert_array_equal(J.jet_score_candidates(m, p, *args)[0], tok)
        J.jet_prefix_free(p)
    finally:
        J.jet_model_free(m)


@pytest.mark.parametrize("dtype", [J.JET_BF16, J.JET_BF16_SINGLE, J.JET_F16P])
def test_modes_without_caches_in_8_bits_are_refused(dtype, model_dir):
    path = jet_synth.ensure_model("small_gqa_bf16", cache_dir=model_dir)
    with pytest.raises(J.JetError) as e:
        J.jet_model_load(path, dtype=dtype, flags=J.JET_FLAG_QCACHE_INT8)
    assert e.value.code == J.JET_E_INVALID
    with pytest.raises(J.JetError) as e:
        J.jet_model_load(path, dtype=J.JET_F16, flags=J.JET_FLAG_QCACHE_INT8 | J.JET_FLAG_QCACHE_E4M3)
    assert e.value.code == J.JET_E_INVALID
