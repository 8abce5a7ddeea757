"""GPU: calls of the operators on device arrays that their documentation allows
and that lie at its edges. Tolerances as in test_gpu_ops.py, by whose helpers
the outputs are compared with the 64-bit references."""
import numpy as np
import pytest
import torch

from paper_2609_33874_amd import jet as J
from test_gpu_ops import case, check_attention, i32, i64, offsets  # noqa: F401

pytestmark = pytest.mark.gpu


def test_workspace_while_the_current_stream_still_writes_a_freed_block():
    """Split keys on another stream: their partials lie apart from memory that queued work is about to write."""
    p, q = case(50, 0, 32, 128, 2, 4, [9000], [1], "f16")
    args, kw = (p.gpu, i64(p.slot0), i32(p.lens), q), dict(max_rows=1, max_len=9000)
    want = J.jet_qcache_attention(*args, torch.empty_like(q), **kw)
    n = J.jet_qcache_attention_workspace(p.gpu, 1, 8, max_len=9000)
    assert n > 0  # split
    st = torch.cuda.Stream()
    out = torch.empty_like(q)
    torch.cuda.synchronize()
    freed = torch.empty(n, dtype=torch.uint8, device="cuda")
    for _ in range(200):
        freed.fill_(255)  # NaN, as f32
    del freed
    J.jet_qcache_attention(*args, out, stream=st.cuda_stream, **kw)
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    # the null stream by its handle, from another current stream
    with torch.cuda.stream(st):
        J.jet_qcache_attention(*args, out.zero_(), stream=st.cuda_stream, **kw)
        st.synchronize()
        assert torch.equal(out, want)
        J.jet_qcache_attention(*args, out, stream=0, **kw)
    torch.cuda.synchronize()
    assert torch.equal(out, want)


@pytest.mark.parametrize("max_rows,max_len", [(1, 10), (1, 5000), (9, 10), (40, 10), (300, 5000)])
def test_an_empty_sequence_behind_a_full_cache(max_rows, max_len):
    """Its slot is the running sum's, n_slots: its rows see no token, wherever in the batch it stands."""
    p, q = case(51, 0, 16, 64, 1, 4, [20, 0, 33], [1, 2, 2], "f16")
    S = p.slots - 16  # without the spare block behind: a cache that its sequences fill
    full = J.QCache(*[t[:, :n].contiguous() for t, n in zip(p.gpu.tensors, (S, S, S // 16, S // 16))], 16, 0)
    assert S == 32 + 48
    for slot0, lens, rows in (([0, 32, 80], [20, 33, 0], [1, 2, 2]), ([80, 0, 32], [0, 20, 33], [2, 1, 2]),
                              ([80], [0], [5]), ([80], [1], [5]), ([96], [0], [5])):
        o, lse = torch.full_like(q, 5.0), torch.full(q.shape[:2], 5.0, device="cuda")
        J.jet_qcache_attention(full, i64(slot0), i32(lens), q, o, row_offsets=i32(offsets(rows)), max_rows=max_rows,
                               max_len=max_len, lse=lse)
        for s, n, (a, b) in zip(slot0, lens, zip(offsets(rows), offsets(rows)[1:])):
            if s > S or s + n > S:  # outside: left as it was
                assert torch.all(o[a:b] == 5.0) and torch.all(lse[a:b] == 5.0)
            elif n == 0:
                assert torch.all(o[a:b] == 0.0) and torch.all(lse[a:b] == -np.inf)
            else:
                assert torch.all(o[a:b] != 5.0) and torch.all(torch.isfinite(lse[a:b]))
        before = [t.clone() for t in full.tensors]
        if max(lens) == 0 or 1 in lens:
            J.jet_qcache_write(full, i64(slot0), i32(lens), q[:, :1], q[:, :1], row_offsets=i32(offsets(rows)))
            k, v = (torch.full((5, 1, 64), 5.0, device="cuda") for _ in "kv")
            J.jet_qcache_read(full, i64(slot0), i32(lens), k, v, row_offsets=i32(offsets(rows)))
            assert torch.all(k == 5.0) and torch.all(v == 5.0)
            assert all(torch.equal(a, b) for a, b in zip(before, full.tensors))
