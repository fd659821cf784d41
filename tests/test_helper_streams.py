"""The helpers that allocate for a call on a given stream do it on that stream."""
import contextlib

import pytest
import torch

import paper_2607_12969_gb300 as lrc
from test_abi import L                     # noqa: F401  (the fixture)


class Recorder:
    """Stands for a stream: what torch does is noted with the stream it was
    asked to do it on."""

    def __init__(self, monkeypatch, *calls):
        self.now, self.seen = None, []
        monkeypatch.setattr(torch.cuda, "stream", self.on)
        monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: ("handle", handle))
        monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: "default")
        for name in ("empty", "zeros"):
            monkeypatch.setattr(torch, name, self.noted(name, getattr(torch, name)))
        for name in calls:
            monkeypatch.setattr(lrc, name, self.noted(name, lambda *a: None))
        monkeypatch.setattr(torch.Tensor, "contiguous", self.noted("contiguous", torch.Tensor.contiguous))

    @contextlib.contextmanager
    def on(self, stream):
        self.now, before = stream, self.now
        yield
        self.now = before

    def noted(self, name, f):
        def g(*a, **k):
            self.seen.append((name, self.now))
            return f(*a, **k)
        return g


@pytest.mark.parametrize("stream,on", [("other", "other"), (7, ("handle", 7)), (0, "default"), (None, None)])
def test_memory_of_a_helper_is_the_streams(L, monkeypatch, stream, on):     # noqa: F811
    W = torch.randn(40, 48).t()                          # not contiguous: copied first
    for call, work in (("lrc_q4_round", lambda: lrc.q4_matrix(W, "f16", 32, True, stream=stream)),
                       ("lrc_round_factors", lambda: lrc.round_matrix(W.double(), "f32", stream=stream)),
                       ("lrc_widen_factors", lambda: lrc.widen_matrix(W, "f32", 40, stream=stream))):
        with monkeypatch.context() as mp:
            r = Recorder(mp, call)
            work()
        assert call in [name for name, _ in r.seen] and len(r.seen) >= 2
        assert all(s == on for _, s in r.seen), (call, r.seen)


@pytest.mark.gpu
def test_a_matrix_rounded_on_another_stream(cuda):
    """With work that the current stream still has to do before what it is asked
    for later: the result on the other stream does not depend on it."""
    lrc.load()
    W = torch.randn((300, 700), device=cuda).t()
    want = lrc.q4_matrix(W, "f16", 64, True)
    torch.cuda.synchronize()
    for other in (torch.cuda.Stream(), torch.cuda.Stream().cuda_stream):
        torch.cuda._sleep(20_000_000)
        got = lrc.q4_matrix(W, "f16", 64, True, stream=other)
        torch.cuda.synchronize()
        for a, b in zip(got[:3], want[:3]):
            assert torch.equal(a, b)
