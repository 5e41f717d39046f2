"""Calls on a stream that is not the current one: what the binding allocates
for them comes from the current stream's memory, which kernels issued there may
still use."""
from types import SimpleNamespace

import pytest
import torch

from paper_2401_11202_amd import partir as P


class FakeStream:
    def __init__(self, handle):
        self.cuda_stream, self.waits = handle, []

    def wait_stream(self, other):
        self.waits.append(other)


class FakeTensor:
    def __init__(self, n):
        self.n, self.device, self.used = n, "cuda:0", []

    def numel(self):
        return self.n

    def record_stream(self, s):
        self.used.append(s)


@pytest.fixture
def here(monkeypatch):
    s = FakeStream(11)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: s)
    return s


def test_another_stream_waits_for_the_memory_it_is_given(here):
    s, t, empty = FakeStream(22), FakeTensor(4), FakeTensor(0)
    P._on_stream(s, None, t, empty)
    assert s.waits == [here] and t.used == [s] and empty.used == []


def test_a_raw_handle_is_a_stream_too(here, monkeypatch):
    made = []
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda h, device: made.append(FakeStream(h)) or made[-1])
    default = FakeStream(0)
    monkeypatch.setattr(torch.cuda, "default_stream", lambda d: default)
    t = FakeTensor(4)
    P._on_stream(33, t)
    assert made[0].cuda_stream == 33 and made[0].waits == [here] and t.used == made
    P._on_stream(0, t)
    assert default.waits == [here] and t.used == made + [default]


def test_nothing_to_do(here):
    t = FakeTensor(4)
    P._on_stream(None, t)
    P._on_stream(11, t)                      # the current stream itself
    P._on_stream(SimpleNamespace(cuda_stream=11), t)
    s = FakeStream(22)
    P._on_stream(s, None, FakeTensor(0))     # nothing was allocated: nothing to wait for
    assert t.used == [] and s.waits == []


@pytest.mark.gpu
@pytest.mark.parametrize("raw", [False, True])
def test_memory_in_use_on_the_current_stream(raw):
    """Outputs and workspaces of calls on another stream while the current one
    still reads freed tensors of their sizes."""
    f = P.rotary_frequencies(128)
    n = 1 << 12
    x = torch.randn(n, 1024, device="cuda").bfloat16()
    g = [torch.randn(n, 1024, device="cuda") for _ in range(3)]
    kw = dict(B=1, Sq=8, Sk=n, n_heads=8)
    calls = [lambda s: P.rotary(x, None, f, d_head=128, stream=s)[0], lambda s: P.cross_attention(x[:8], x, x, stream=s, **kw),
             lambda s: P.grad_norm(g, stream=s)]
    want = [c(None) for c in calls]
    busy = torch.randn(1 << 27, device="cuda")
    for call, ref in zip(calls, want):
        s = torch.cuda.Stream()
        for size in (n * 1024, 8 * 1024, n * 1024 // 4):
            src = torch.randn(size, device="cuda").bfloat16()
            torch.cuda.synchronize()
            old = src.clone()
            for _ in range(8):
                busy.mul_(1.0)
            seen = old.clone()               # still waits behind the work above
            del old
            got = call(s.cuda_stream if raw else s)
            torch.cuda.synchronize()
            assert torch.equal(seen, src) and torch.equal(got, ref)
