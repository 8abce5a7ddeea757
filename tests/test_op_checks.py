"""Refusals of the operators on device arrays, without a GPU: every argument
that the host can see is checked before anything touches a device. The
pointers here are never followed."""
import ctypes

import pytest

from paper_2609_33874_amd import jet as J

A = 0x10000  # an aligned address that is not memory


def cache(**over):
    d = dict(format=J.JET_QCACHE_INT8, block=32, n_heads=2, head_dim=128, n_slots=64, k=A, v=A, k_exp=A, v_exp=A)
    return J.jet_qcache(**dict(d, **over))


def batch(**over):
    d = dict(n_seq=2, n_rows=3, max_rows=2, reserved=0, max_len=40, slot0=A, len=A, row_offsets=A)
    return J.jet_qcache_batch(**dict(d, **over))


def rows(**over):
    return J.jet_rows(**dict(dict(p=A, type=J.JET_T_F16, reserved=0, row_stride=256, head_stride=128), **over))


def call(fn, *args):
    got = getattr(J.lib(), fn)(*[ctypes.byref(a) if isinstance(a, ctypes.Structure) else a for a in args])
    return got, J.jet_last_error()


def write(c, b, k, v):
    return call("jet_qcache_write", c, b, k, v, None)


def read(c, b, k, v):
    return call("jet_qcache_read", c, b, k, v, None)


def attention(c, b, q, o, heads=4, scale=0.1, causal=1, lse=None, ws=A, ws_n=1 << 40):
    return call("jet_qcache_attention", c, b, heads, scale, causal, q, o, lse, ws, ws_n, None)


BAD_CACHES = [dict(format=2), dict(format=-1), dict(block=0), dict(block=24), dict(block=256), dict(n_heads=0),
              dict(n_heads=1025), dict(head_dim=32), dict(head_dim=96), dict(n_slots=63), dict(n_slots=-32),
              dict(n_slots=1 << 41), dict(k=None), dict(v=None), dict(k_exp=None), dict(v_exp=None), dict(k=A + 8),
              dict(v=A + 1)]
BAD_BATCHES = [dict(n_seq=-1), dict(n_seq=65536), dict(n_rows=-1), dict(n_rows=(1 << 30) + 1), dict(max_rows=-1),
               dict(max_len=-1), dict(slot0=None), dict(len=None), dict(row_offsets=None, n_rows=1), dict(slot0=A + 4),
               dict(len=A + 2), dict(row_offsets=A + 1)]
BAD_ROWS = [dict(type=3), dict(type=-1), dict(p=None), dict(p=A + 1), dict(row_stride=-1), dict(head_stride=-1),
            dict(row_stride=1 << 41)]


@pytest.mark.parametrize("over", BAD_CACHES)
def test_bad_caches(over):
    for got, msg in (write(cache(**over), batch(), rows(), rows()), read(cache(**over), batch(), rows(), rows()),
                     attention(cache(**over), batch(), rows(), rows())):
        assert got == J.JET_E_INVALID and "cache" in msg


@pytest.mark.parametrize("over", BAD_BATCHES)
def test_bad_batches(over):
    for got, msg in (write(cache(), batch(**over), rows(), rows()), read(cache(), batch(**over), rows(), rows()),
                     attention(cache(), batch(**over), rows(), rows())):
        assert got == J.JET_E_INVALID and msg


@pytest.mark.parametrize("over", BAD_ROWS)
def test_bad_rows(over):
    for got, msg in (write(cache(), batch(), rows(**over), rows()), write(cache(), batch(), rows(), rows(**over)),
                     read(cache(), batch(), rows(**over), rows()), read(cache(), batch(), rows(), rows(**over)),
                     attention(cache(), batch(), rows(**over), rows()),
                     attention(cache(), batch(), rows(), rows(**over))):
        assert got == J.JET_E_INVALID and msg


def test_null_structs():
    n = None
    for got, _ in (write(n, batch(), rows(), rows()), write(cache(), n, rows(), rows()),
                   write(cache(), batch(), n, rows()), read(cache(), batch(), rows(), n),
                   attention(cache(), batch(), n, rows()), attention(cache(), batch(), rows(), n),
                   call("jet_logits_adjust", n, n)):
        assert got == J.JET_E_INVALID


def test_types_and_strides_of_written_rows():
    f32 = dict(type=J.JET_T_F32)
    for got, _ in (write(cache(), batch(), rows(), rows(**f32)),                   # k and v of different types
                   read(cache(), batch(), rows(row_stride=0), rows()),             # rows on top of each other
                   read(cache(), batch(), rows(), rows(head_stride=0)),
                   attention(cache(), batch(), rows(**f32), rows()),               # no f32 queries
                   attention(cache(), batch(), rows(), rows(type=J.JET_T_BF16)),   # q's type or f32
                   attention(cache(), batch(), rows(), rows(row_stride=0))):
        assert got == J.JET_E_INVALID


def test_attention_arguments():
    for over in (dict(heads=0), dict(heads=3), dict(heads=130), dict(scale=float("nan")), dict(scale=float("inf")),
                 dict(causal=2), dict(causal=-1), dict(lse=A + 2)):
        got, msg = attention(cache(), batch(), rows(), rows(), **over)
        assert got == J.JET_E_INVALID and msg, over


def test_attention_of_too_many_heads_and_rows():
    q = rows(row_stride=1 << 20)
    got, msg = attention(cache(n_heads=1024), batch(), q, q, heads=32768 + 1024)
    assert got == J.JET_E_INVALID and "heads" in msg
    got, msg = attention(cache(n_heads=1), batch(n_rows=1 << 30), q, q, heads=2)
    assert got == J.JET_E_INVALID and "n_rows" in msg


def workspace(c, b, heads):
    n = ctypes.c_int64(-1)
    got, _ = call("jet_qcache_attention_workspace", c, b, heads, ctypes.byref(n))
    return got, n.value


def test_workspace_size_and_refusals():
    assert workspace(cache(n_heads=0), batch(), 4)[0] == J.JET_E_INVALID
    assert workspace(cache(), batch(n_seq=-1), 4)[0] == J.JET_E_INVALID
    assert workspace(cache(), batch(), 3)[0] == J.JET_E_INVALID
    assert call("jet_qcache_attention_workspace", cache(), batch(), 4, None)[0] == J.JET_E_INVALID
    # the device arrays are not needed, and the call itself takes a workspace of that size and no smaller
    for n_seq, max_len in ((1, 100), (1, 100000), (64, 4096), (1000, 64)):
        c = cache(n_heads=8, n_slots=1 << 24)
        b = batch(n_seq=n_seq, n_rows=n_seq, max_rows=1, max_len=max_len, row_offsets=None)
        got, n = workspace(c, batch(n_seq=n_seq, n_rows=n_seq, max_rows=1, max_len=max_len, slot0=None, len=None,
                                    row_offsets=None), 40)
        assert got == J.JET_OK and n >= 0
        if n:
            q = rows(row_stride=40 * 128)
            for ws, size in ((A, n - 1), (None, n), (A + 4, n)):
                got, msg = attention(c, b, q, q, heads=40, ws=ws, ws_n=size)
                assert got == J.JET_E_INVALID and "workspace" in msg


def logits(**over):
    d = dict(n_rows=2, vocab=100, type=J.JET_T_F32, n_masks=2, logits=A, out=A, row_stride=100, out_stride=100,
             hist_offsets=A, hist_ids=A, hist_prompt=A, n_hist=5, repetition=A, presence=A, frequency=A,
             bias_offsets=A, bias_ids=A, bias_values=A, n_bias=3, masks=A, mask_stride=4, mask_index=A)
    return J.jet_logits_args(**dict(d, **over))


@pytest.mark.parametrize("over", [
    dict(n_rows=-1), dict(n_rows=(1 << 20) + 1), dict(vocab=0), dict(vocab=(1 << 24) + 1), dict(type=3),
    dict(logits=None), dict(out=None), dict(logits=A + 2), dict(out=A + 1), dict(row_stride=99), dict(out_stride=99),
    dict(out_stride=101), dict(n_hist=-1), dict(n_hist=(1 << 30) + 1), dict(n_bias=(1 << 30) + 1), dict(hist_ids=None), dict(n_bias=-1),
    dict(bias_ids=None), dict(bias_values=None), dict(n_masks=-1), dict(mask_stride=3), dict(masks=None),
    dict(mask_index=None, n_masks=1), dict(hist_offsets=A + 2), dict(repetition=A + 1), dict(masks=A + 2)])
def test_bad_logits(over):
    got, msg = call("jet_logits_adjust", logits(**over), None)
    assert got == J.JET_E_INVALID and msg


def test_calls_without_work_succeed():
    """No sequence, no row: nothing to do, on any machine."""
    none = dict(n_seq=0, n_rows=0, slot0=None, len=None, row_offsets=None)
    empty = dict(p=None)
    assert write(cache(), batch(**none), rows(**empty), rows(**empty))[0] == J.JET_OK
    assert read(cache(), batch(**none), rows(**empty), rows(**empty))[0] == J.JET_OK
    assert attention(cache(), batch(**none), rows(**empty), rows(**empty))[0] == J.JET_OK
    assert call("jet_logits_adjust", logits(n_rows=0, logits=None, out=None), None)[0] == J.JET_OK


def test_a_good_call_clears_the_message():
    assert write(None, batch(), rows(), rows())[0] == J.JET_E_INVALID and J.jet_last_error()
    none = dict(n_seq=0, n_rows=0, slot0=None, len=None, row_offsets=None)
    assert write(cache(), batch(**none), rows(), rows())[0] == J.JET_OK and J.jet_last_error() == ""
