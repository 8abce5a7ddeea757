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
