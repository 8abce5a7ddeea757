"""GPU: traces whose logits leave nothing to sample, and rules at their edges."""
import numpy as np
import pytest

import jet_synth
from paper_2609_33874_amd import jet as J

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def nan_model(tmp_path_factory):
    """A model whose every logit is NaN."""
    path = str(tmp_path_factory.mktemp("nan") / "nan.jetm")
    header = jet_synth.write_model(path, "small_gqa_bf16")
    t = next(t for t in header["tensors"] if t["name"] == "final_norm")
    w = np.memmap(path, dtype=np.float32, mode="r+", offset=t["offset"], shape=tuple(t["shape"]))
    w[:] = np.nan
    w.flush()
    return path


@pytest.mark.parametrize("flags", [0, J.JET_FLAG_QCACHE_INT8])
@pytest.mark.parametrize("dtype", [J.JET_FP32, J.JET_F16])
@pytest.mark.parametrize("rules", [False, True])
def test_logits_that_are_not_numbers_end_the_trace(dtype, flags, rules, nan_model):
    """No token is found (-1), at the first of several steps: the call fails and later steps read no embedding of it."""
    wl = jet_synth.make_workload("small", n_questions=2)
    m = J.jet_model_load(nan_model, dtype=dtype, flags=flags)
    try:
        p = J.jet_prefill_prefix(m, wl.prefix_offsets, wl.prefix_tokens)
        with pytest.raises(J.JetError) as e:
            if rules:
                J.jet_generate_trace_rules(m, p, 2, 3, 0.7, 1, repetition=1.2)
            else:
                J.jet_generate_trace(m, p, 2, 3, 0.7, 1)
        assert e.value.code == J.JET_E_DEVICE and "finite" in str(e.value)
        J.jet_prefix_free(p)
    finally:
        J.jet_model_free(m)


@pytest.mark.parametrize("tau", [0.0, 0.8])
@pytest.mark.parametrize("flags", [0, J.JET_FLAG_QCACHE_INT8])
def test_a_forbidden_token_is_never_sampled(flags, tau, model_dir):
    """One allowed token whose penalty overflows at its third time: the step has no token, not the lowest forbidden one."""
    path = jet_synth.ensure_model("small_gqa_bf16", cache_dir=model_dir)
    wl = jet_synth.make_workload("small", n_questions=2)
    words = np.zeros((1, (3000 + 31) // 32), np.uint32)
    words[0, 17 // 32] = 1 << 17 % 32
    m = J.jet_model_load(path, dtype=J.JET_F16, flags=flags)
    try:
        for n in (2, 4):
            p = J.jet_prefill_prefix(m, wl.prefix_offsets, wl.prefix_tokens)
            kw = dict(frequency=2e38, masks=words, mask_index=np.zeros((2, n), np.int32))
            if n == 2:
                assert np.all(J.jet_generate_trace_rules(m, p, 2, n, tau, 3, **kw) == 17)
            else:
                with pytest.raises(J.JetError) as e:
                    J.jet_generate_trace_rules(m, p, 2, n, tau, 3, **kw)
                assert e.value.code == J.JET_E_DEVICE and "finite" in str(e.value)
            J.jet_prefix_free(p)
    finally:
        J.jet_model_free(m)


def test_mask_indices_without_masks(model_dir):
    """Steps that name a mask are refused where there is none; steps that name none run as without rules."""
    path = jet_synth.ensure_model("small_gqa_bf16", cache_dir=model_dir)
    wl = jet_synth.make_workload("small", n_questions=2)
    none = np.zeros((0, (3000 + 31) // 32), np.uint32)
    m = J.jet_model_load(path, dtype=J.JET_F16)
    try:
        p = J.jet_prefill_prefix(m, wl.prefix_offsets, wl.prefix_tokens)
        for masks in (None, none):
            for index in (np.zeros((2, 3), np.int32), np.array([[-1, -1, -1], [-1, -1, 0]], np.int32)):
                with pytest.raises(J.JetError) as e:
                    J.jet_generate_trace_rules(m, p, 2, 3, 0.0, 0, masks=masks, mask_index=index)
                assert e.value.code == J.JET_E_INVALID and "mask" in str(e.value)
        got = J.jet_generate_trace_rules(m, p, 2, 3, 0.0, 0, mask_index=np.full((2, 3), -1, np.int32))
        J.jet_prefix_free(p)
        p = J.jet_prefill_prefix(m, wl.prefix_offsets, wl.prefix_tokens)
        np.testing.assert_array_equal(got, J.jet_generate_trace(m, p, 2, 3))
        J.jet_prefix_free(p)
    finally:
        J.jet_model_free(m)


@pytest.mark.parametrize("flags", [0, J.JET_FLAG_QCACHE_INT8])
def test_a_refused_context_leaves_no_memory_behind(flags, model_dir):
    import torch
    path = jet_synth.ensure_model("small_gqa_bf16", cache_dir=model_dir)
    n_q = 1025
    wl = jet_synth.from_lists([np.array([q % 3000], np.int32) for q in range(n_q)],
                              [[np.array([1], np.int32)] for _ in range(n_q)])
    off = np.full(n_q + 1, (1 << 20) - 1, np.int64)
    off[0] = 0
    m = J.jet_model_load(path, dtype=J.JET_F16, flags=flags)
    try:
        p = J.jet_prefill_prefix(m, wl.prefix_offsets, wl.prefix_tokens)
        free = []
        for _ in range(4):
            with pytest.raises(J.JetError) as e:
                J.jet_generate_trace_rules(m, p, n_q, 1, context=(off, np.zeros(off[-1], np.int32)))
            assert e.value.code == J.JET_E_INVALID
            torch.cuda.synchronize()
            free.append(torch.cuda.mem_get_info()[0])
        assert len(set(free)) == 1, free
        J.jet_prefix_free(p)
    finally:
        J.jet_model_free(m)


@pytest.mark.parametrize("flags", [0, J.JET_FLAG_QCACHE_INT8])
def test_a_trace_too_long_for_the_memory_leaves_room_for_a_shorter_one(flags, model_dir):
    """JET_E_OOM changes nothing: what had been allocated until then is given back."""
    path = jet_synth.ensure_model("small_gqa_bf16", cache_dir=model_dir)
    wl = jet_synth.make_workload("small", n_questions=8)
    short = 2 ** 21 // (8 * 2 * 128 * (1 if flags else 2))  # four buffers of 2 MiB; of a long one the first fits there
    args = (wl.q_cand_offsets, wl.cand_tok_offsets, wl.cand_tokens)

    def load(budget):
        m = J.jet_model_load(path, dtype=J.JET_F16, flags=flags, max_device_bytes=budget)
        p = J.jet_prefill_prefix(m, wl.prefix_offsets, wl.prefix_tokens)
        J.jet_score_candidates(m, p, *args)
        return m, p

    # the least budget under which the short trace runs, to 1 MiB
    lo, hi = 0, 256
    while hi - lo > 1:
        mid = (lo + hi) // 2
        try:
            m, p = load(mid << 20)
        except J.JetError:
            lo = mid
            continue
        try:
            J.jet_generate_trace(m, p, 8, short)
            hi = mid
        except J.JetError as e:
            assert e.code == J.JET_E_OOM
            lo = mid
        J.jet_prefix_free(p)
        J.jet_model_free(m)
    m, p = load(hi << 20)
    tok, _ = J.jet_score_candidates(m, p, *args)
    for _ in range(2):
        with pytest.raises(J.JetError) as e:
            J.jet_generate_trace(m, p, 8, 3 * short)
        assert e.value.code == J.JET_E_OOM
    np.testing.assert_array_equal(J.jet_score_candidates(m, p, *args)[0], tok)
    J.jet_generate_trace(m, p, 8, short)
    J.jet_prefix_free(p)
    J.jet_model_free(m)
