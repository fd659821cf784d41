"""Distillation of logits far from zero, and of rows that hold only the type's
lowest number: a softmax does not depend on an offset of its logits."""
import math

import pytest
import torch

import layer_ref as R
from layer_ref import OUT_TINY, OUT_U, STORE, U

pytestmark = pytest.mark.gpu

TINY = 2.0 ** -125       # what is smaller may be flushed to 0 by the exponentials


def inputs(dev, rows, V, K, fmt, offset, seed):
    gen = torch.Generator(device=dev).manual_seed(seed)
    z = (torch.randn((rows, V), generator=gen, device=dev) * 2 + offset).to(STORE[fmt])
    idx = torch.randint(0, V, (rows, K), generator=gen, device=dev)
    t = torch.randn((rows, K), generator=gen, device=dev) * 2 + offset
    w = torch.rand(rows, generator=gen, device=dev) + 0.5
    return z, t, idx, w


def errors(z, t, idx, w, tau, want, out):
    """Bounds that know the logits only by their distances d from the row's largest,
    over tau.  A term's exponent is off by 3 U d (the factor log2(e) / tau by 2 U, a
    rounding), exp2 by 4 U, the sum by V / 256 + 40 roundings; the mean of d under the
    softmax is at most ln V.  The teacher's likewise with K / 32 + 40."""
    loss, lse, dz, ps = want
    V, K = z.shape[1], t.shape[1]
    d = (z.double().amax(1, keepdim=True) - z.double()) / tau
    bl = (V / 256 + 44 + 3 * math.log(V)) * U
    dt = (t.double().amax(1, keepdim=True) - t.double()) / tau
    bp = (K / 32 + 48 + 3 * math.log(K + 1) + 4 * dt) * U                    # of p_k, relative; of log p_k, absolute
    logp = torch.log(ps)
    logq = (z.double() / tau - lse[:, None]).gather(1, idx)
    dq = d.gather(1, idx)
    each = 2 * bp + 2 * bl + 4 * U * (dq + logq.abs() + logp.abs()) + bp * (logp - logq).abs()
    b_loss = tau ** 2 * w.double() * (ps * each).sum(1) * 1.01 + (K / 32 + 12) * U * \
        tau ** 2 * w.double() * (ps * (logp - logq).abs()).sum(1)
    b_lse = 2 * bl + 2 * U * lse.abs()
    c = (tau * w.double())[:, None]
    q = torch.exp(z.double() / tau - lse[:, None])
    p = torch.zeros_like(q).scatter_add_(1, idx, ps)
    pb = torch.zeros_like(q).scatter_add_(1, idx, ps * bp)
    b_dz = c * (q * (2 * bl + (12 + 4 * d) * U) + pb + 8 * U * p + TINY) + OUT_U[out] * dz.abs() * 1.01 + OUT_TINY[out]
    return b_loss, b_lse, b_dz


def from_lse(z, t, idx, w, lse, tau, ps, out):
    """The gradient by its definition with the lse as it is given, whose rounding is
    not the call's, and a bound: the distance d of a logit from it, over tau, is off by
    4 U of itself."""
    K = t.shape[1]
    d = z.double() / tau - lse.double()[:, None]
    q = torch.exp(d)
    p = torch.zeros_like(q).scatter_add_(1, idx, ps)
    dt = (t.double().amax(1, keepdim=True) - t.double()) / tau
    pb = torch.zeros_like(q).scatter_add_(1, idx, ps * ((K / 32 + 48 + 3 * math.log(K + 1) + 4 * dt) * U))
    c = (tau * w.double())[:, None]
    want = c * (q - p)
    bound = c * (q * (16 + 4 * d.abs()) * U + pb + 8 * U * p + TINY)
    return want, bound + OUT_U[out] * want.abs() * 1.01 + OUT_TINY[out]


@pytest.mark.parametrize("rows,V,K", [(5, 640, 7), (3, 5000, 32), (2, 40001, 9), (1, 150001, 64), (700, 700, 5)])
@pytest.mark.parametrize("fmt,tau", [("f32", 1.0), ("f32", 0.7), ("f16", 2.0), ("bf16", 0.1)])
@pytest.mark.parametrize("offset", [0.0, 100.0, -3000.0])
def test_an_offset_changes_nothing(lrc, cuda, rows, V, K, fmt, tau, offset):
    z, t, idx, w = inputs(cuda, rows, V, K, fmt, offset, rows + V)
    loss, lse = torch.empty(rows, device=cuda), torch.empty(rows, device=cuda)
    dz = torch.empty_like(z)
    tail = (rows, V, K, V, K, V, tau, fmt, "f32")
    lrc.lrc_distill(z, t, idx, w, loss, lse, dz, *tail)
    tau = float(torch.tensor(tau))                       # the binary32 number that the call takes
    want = R.distill(z, t, idx, w, tau)
    b_loss, b_lse, b_dz = errors(z, t, idx, w, tau, want, STORE[fmt])
    R.within(lse, want[1], b_lse, "lse")
    R.within(dz, want[2], b_dz, "dz")
    R.within(loss, want[0], b_loss, "loss")


@pytest.mark.parametrize("rows,V,K", [(5, 640, 7), (2, 40001, 9), (1, 150001, 64), (700, 700, 5)])
@pytest.mark.parametrize("fmt,tau", [("f32", 1.0), ("f32", 0.7), ("f16", 2.0), ("bf16", 0.1)])
@pytest.mark.parametrize("offset", [0.0, 100.0, -3000.0])
def test_gradient_from_a_given_sum(lrc, cuda, rows, V, K, fmt, tau, offset):
    z, t, idx, w = inputs(cuda, rows, V, K, fmt, offset, rows + V + 1)
    given = torch.logsumexp(z.double() / float(torch.tensor(tau)), 1).float()
    dz = torch.empty_like(z)
    lrc.lrc_distill_grad(z, t, idx, w, given, None, dz, rows, V, K, V, K, V, tau, fmt, "f32")
    tau = float(torch.tensor(tau))
    want, bound = from_lse(z, t, idx, w, given, tau, R.distill(z, t, idx, w, tau)[3], STORE[fmt])
    R.within(dz, want, bound)


@pytest.mark.parametrize("rows,V", [(4, 50), (4, 9000), (2, 40001), (200, 3000), (2, 300001)])
@pytest.mark.parametrize("fmt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("tau", [1.0, 0.5, 2.0])
def test_rows_of_the_lowest_number(lrc, cuda, rows, V, fmt, tau):
    """A row whose mask leaves nothing, in the form of the type's lowest number:
    all logits are equal, q = 1 / V.  In other rows that number has q = 0."""
    K, dt = 6, STORE[fmt]
    low = torch.finfo(dt).min
    z, t, idx, w = inputs(cuda, rows, V, K, fmt, 0.0, V)
    z[1] = low
    z[0, ::3] = low
    idx[0] = 1 + 3 * torch.arange(K, device=cuda)        # places that are not masked
    loss, lse = torch.empty(rows, device=cuda), torch.empty(rows, device=cuda)
    dz = torch.empty_like(z)
    lrc.lrc_distill(z, t, idx, w, loss, lse, dz, rows, V, K, V, K, V, tau, fmt, "f32")
    seen = z.double().clone()
    seen[1] = 0                                          # an offset
    seen[0, ::3] = -math.inf
    want = R.distill(seen, t, idx, w, tau)
    finite = torch.where(torch.isfinite(seen), seen, seen[:, 1:2])
    b_loss, _, b_dz = errors(finite, t, idx, w, tau, (want[0], want[1], want[2], want[3]), dt)
    R.within(loss, want[0], b_loss, "loss")
    R.within(dz, want[2], b_dz, "dz")
    exact = torch.tensor([low / tau + math.log(V)], dtype=torch.float64, device=cuda)
    if abs(low / tau) >= 2.0 ** 128:                     # no binary32 number
        assert float(lse[1]) == -math.inf
        return
    R.within(lse[1:2], exact, 2 * U * exact.abs(), "lse")
    # apart: exp(z / tau - lse) of the lse as it is, although log V is lost in it
    lrc.lrc_distill_grad(z, t, idx, w, lse, None, dz, rows, V, K, V, K, V, tau, fmt, "f32")
    one = slice(1, 2)
    apart, bound = from_lse(z[one], t[one], idx[one], w[one], lse[one], tau, want[3][one], dt)
    R.within(dz[one], apart, bound, "dz apart")
