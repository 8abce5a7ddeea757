"""The Python side of the operators on device arrays, without a GPU: the library
and torch's streams are stand-ins that record what they are asked for."""
import contextlib
import types

import pytest
import torch

from paper_2609_33874_amd import jet as J


class Streams:
    """Enough of torch for the binding: which stream is current when memory is allocated."""

    def __init__(self, current):
        self.current, self.allocated_on = current, []
        self.uint8, self.int32, self.int64, self.float32 = torch.uint8, torch.int32, torch.int64, torch.float32
        self.cuda = types.SimpleNamespace(stream=self.use, ExternalStream=self.external, default_stream=lambda device: 0)

    @staticmethod
    def external(ptr, device):
        assert ptr, "a null handle makes a new stream"
        return ptr

    @contextlib.contextmanager
    def use(self, s):
        before, self.current = self.current, s
        yield
        self.current = before

    def empty(self, n, dtype, device):
        self.allocated_on.append(self.current)
        return torch.empty(n, dtype=dtype)


class Lib:
    def __init__(self):
        self.launched_on = []

    def jet_qcache_attention_workspace(self, c, b, heads, out):
        out.value = 4096
        return J.JET_OK

    def jet_qcache_attention(self, *args):
        self.launched_on.append(args[-1])
        return 0


@pytest.mark.parametrize("current", [0, 7])
@pytest.mark.parametrize("stream", [None, 0, 7, 9])
def test_a_workspace_belongs_to_the_stream_that_uses_it(monkeypatch, stream, current):
    """Memory that the current stream freed may still be in use there: another stream's call must not get it."""
    fake, lib = Streams(current), Lib()
    kinds = {torch.float32: J.JET_T_F32, torch.float16: J.JET_T_F16, torch.bfloat16: J.JET_T_BF16}
    monkeypatch.setattr(J, "_torch", (fake, kinds, lambda device: fake.current))
    monkeypatch.setattr(J, "lib", lambda: lib)
    cache = types.SimpleNamespace(device=-1, c=J.jet_qcache(0, 32, 2, 64, 64))  # (CPU tensors are on "GPU" -1)
    q = torch.zeros((1, 2, 64), dtype=torch.float16)
    J.jet_qcache_attention(cache, torch.zeros(1, dtype=torch.int64), torch.ones(1, dtype=torch.int32), q,
                           torch.empty_like(q), stream=stream)
    assert lib.launched_on == fake.allocated_on == [current if stream is None else stream]
    assert fake.current == current
