"""The compressed layer of examples/: its operators together, as a program uses
them, each step against the same model in plain torch."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("compressed_layer", os.path.join(ROOT, "examples", "compressed_layer.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_compensation_and_repair(lrc, cuda, example):
    err, losses = example.main(steps=30)
    assert err[1] < err[0]                       # the factors compensate the codes
    assert losses[-1] < losses[0]                # the norm's repair lowers the loss


def test_a_training_step_is_the_gradient_of_its_loss(lrc, cuda, example):
    """Loss and gradients of one step against binary64 autograd of the same
    frozen layer output and head factors.  The chain is binary32: each of its
    five calls is within about 1e-5 of its result (the tolerance of lrc_apply in
    binary32), and the relative errors of such a chain add up."""
    torch.manual_seed(0)
    m, n, V, rows, k, hk = 96, 160, 500, 24, 8, 64
    W, head = torch.randn((m, n), device=cuda) / n ** 0.5, torch.randn((V, m), device=cuda) * (3 / m ** 0.5)
    X = torch.zeros((rows, lrc.lrc_packed_ld(n)), dtype=torch.float16, device=cuda)
    X[:, :n] = torch.randn((rows, n), device=cuda)
    layer = example.Layer(W, k)
    heads = example.factors(head, hk, "f32")
    t = torch.topk(torch.randn((rows, V), device=cuda) * 2, 12, dim=1)
    r = example.Repair(layer, heads, V, hk, t.values.contiguous(), t.indices, X, tau=1.5)
    r.gamma.add_(0.1 * torch.randn(m, device=cuda))
    gamma, beta = (p.double().clone().requires_grad_() for p in (r.gamma, r.beta))
    loss = r.step(0.0)
    U, S, Vt = (f.double() for f in heads[0])
    N = torch.nn.functional.layer_norm(r.H.double(), (m,), gamma, beta, 1e-5)
    Z = ((N @ Vt[:, :m].t()) * S[0, :hk]) @ U[:, :hk].t()
    logp = torch.log_softmax(t.values.double() / 1.5, 1)
    logq = torch.log_softmax(Z / 1.5, 1).gather(1, t.indices)
    want = 1.5 ** 2 * (logp.exp() * (logp - logq)).sum() / rows
    want.backward()
    assert abs(loss - float(want.detach())) <= 5e-5 * float(want.detach())
    for got, p in zip(r.grads, (gamma, beta)):
        assert float((got.double() - p.grad).norm()) <= 5e-5 * float(p.grad.norm())
