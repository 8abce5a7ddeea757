"""GPU: candidate scoring over retained caches in 8 bits at head sizes and group
widths that the other tests' models do not have. Tolerances as in
test_gpu_qcache.py."""
import numpy as np
import pytest

import jet_synth
from oracle.model import Model
from paper_2609_33874_amd import jet as J
from test_gpu_parity import TOL
from test_gpu_qcache import FLAGS, SLACK, oracle_scores, scores

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def models(tmp_path_factory):
    made = {}

    def get(head_dim, n_heads, n_kv_heads):
        key = (head_dim, n_heads, n_kv_heads)
        if key not in made:
            path = str(tmp_path_factory.mktemp("heads") / "{}_{}_{}.jetm".format(*key))
            jet_synth.write_model(path, dict(jet_synth.MODEL_SPECS["small_gqa_bf16"], head_dim=head_dim, n_heads=n_heads,
                                             n_kv_heads=n_kv_heads))
            made[key] = path
        return made[key]
    return get


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("head_dim,n_heads,n_kv_heads", [(64, 8, 2), (64, 4, 4), (128, 2, 2), (64, 32, 1)])
def test_own_rows_of_other_heads(head_dim, n_heads, n_kv_heads, fmt, models):
    """Blocks of 64 and of 128 slots, candidates longer than a key tile; JET_F16 and JET_FP32 against the oracle."""
    path = models(head_dim, n_heads, n_kv_heads)
    rng = np.random.default_rng(60)
    wl = jet_synth.from_lists([rng.integers(0, 3000, size=n).astype(np.int32) for n in (90, 33, 1)],
                              [[rng.integers(0, 3000, size=n).astype(np.int32) for n in lens]
                               for lens in ([70, 1, 9, 66], [3, 2], [5, 20, 20, 20])])
    plain, quant = oracle_scores(Model(path), wl, fmt)
    d_q = np.abs(quant - plain).max()
    got = {}
    for dtype in (J.JET_FP32, J.JET_F16):
        m = J.jet_model_load(path, dtype=dtype, flags=FLAGS[fmt])
        try:
            got[dtype] = scores(m, wl)[0]
            again = scores(m, wl.subset([2]))[0]  # by itself
        finally:
            J.jet_model_free(m)
        assert np.abs(got[dtype] - quant).max() <= TOL[dtype][0] + SLACK[dtype] * d_q
        if dtype == J.JET_F16:
            assert np.abs(again - got[dtype][-len(again):]).max() <= TOL[dtype][0] + SLACK[dtype] * d_q
