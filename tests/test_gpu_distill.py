"""Distillation loss and gradient on the GPU against binary64."""
import math

import pytest
import torch

import layer_ref as R
from layer_ref import OUT_TINY, OUT_U, STORE, U

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


def case(dev, rows, V, K, fmt, tfmt, seed, pad=0, shift=0, holes=True):
    """Logits, teacher entries and weights: absent entries, rows without any,
    rows without weight, masked logits, places named twice."""
    gen = torch.Generator(device=dev).manual_seed(seed)
    z, zb = R.framed((rows, V), STORE[fmt], dev, V + pad, shift=shift)
    z.copy_(torch.randn((rows, V), generator=gen, device=dev) * 2)
    t = (torch.randn((rows, K), generator=gen, device=dev) * 2).to(STORE[tfmt])
    idx = torch.randint(0, V, (rows, K), generator=gen, device=dev)
    w = torch.rand(rows, generator=gen, device=dev) + 0.5
    if holes:
        idx[torch.rand((rows, K), generator=gen, device=dev) < 0.2] = -1
        idx[torch.rand((rows, K), generator=gen, device=dev) < 0.05] = V
        t[torch.rand((rows, K), generator=gen, device=dev) < 0.1] = -INF
        if rows > 2:
            idx[1] = -5
            w[2] = 0
        if V > 100:
            shut = torch.arange(V, device=dev) % 97 == 5
            z[:, shut] = -INF
            idx[(idx >= 0) & (idx % 97 == 5)] = 1
    return z, zb, t, idx, w


def bounds(z, t, idx, w, tau, want, g, out):
    """lse: a sum over at least 256 partial sums; exp(x) within 2 U and the
    error of x, whose parts are rounded at the size of z / tau."""
    loss, lse, dz, ps = want
    V, K = z.shape[1], t.shape[1]
    zf = torch.where(torch.isfinite(z), z, torch.zeros_like(z)).double().abs().amax(1) / tau
    tf = torch.where(torch.isfinite(t), t, torch.zeros_like(t)).double().abs().amax(1) / tau
    top = zf + torch.where(torch.isfinite(lse), lse.abs(), torch.zeros_like(lse))
    bl = (V / 256 + 40 + 8 * top) * U
    bt = (K / 32 + 40 + 8 * tf) * U
    bloss = tau ** 2 * w.double() * (2 * bl + bt * (2 + 2 * tf + 2 * top)) + 2 * U * loss.abs()
    c = (tau * w.double() * g.double())[:, None]
    q = torch.exp(z.double() / tau - lse[:, None])
    p = torch.zeros_like(q)
    p.scatter_add_(1, idx.clamp(0, V - 1), ps)
    want_dz = dz * g.double()[:, None]
    bdz = c * (q * (2 * bl[:, None] + 8 * U) + p * (2 * bt[:, None] + 8 * U)) + OUT_U[out] * want_dz.abs() * 1.01 + OUT_TINY[out]
    return bloss, bl, want_dz, bdz


SHAPES = [(1, 1, 1), (2, 3, 2), (5, 33, 7), (4, 255, 16), (3, 1000, 64), (6, 4096, 32), (2, 32768, 50), (3, 50001, 17),
          (1, 131071, 256), (2, 262144, 9), (1, 600007, 5), (300, 640, 8), (9, 2000, 1024)]


@pytest.mark.parametrize("rows,V,K", SHAPES)
@pytest.mark.parametrize("fmt,tfmt,tau", [("f32", "f32", 1.0), ("f16", "f16", 2.0), ("bf16", "f32", 0.5),
                                          ("f16_o16", "bf16", 4.0)])
@pytest.mark.parametrize("pad,shift", [(0, 0), (3, 1)])
def test_loss_and_gradient(lrc, cuda, rows, V, K, fmt, tfmt, tau, pad, shift):
    z, zb, t, idx, w = case(cuda, rows, V, K, fmt, tfmt, rows + V, pad, shift)
    dz, dzb = R.framed((rows, V), STORE[fmt], cuda, V + 2 * pad, shift=shift)
    loss, lse = (torch.full((rows,), NAN, device=cuda) for _ in range(2))
    tail = (rows, V, K, V + pad, K, V + 2 * pad, tau, fmt, tfmt)
    lrc.lrc_distill(z, t, idx, w, loss, lse, dz, *tail)
    want = R.distill(z, t, idx, w, tau)
    one = torch.ones(rows, device=cuda)
    bloss, bl, want_dz, bdz = bounds(z, t, idx, w, tau, want, one, STORE[fmt])
    R.within(lse, want[1], bl, "lse")
    R.within(loss, want[0], bloss, "loss")
    R.within(dz, want_dz, bdz, "dz")
    R.frame_kept(dz, dzb)
    # forward alone: the same bits
    l2, s2 = (torch.full((rows,), NAN, device=cuda) for _ in range(2))
    lrc.lrc_distill(z, t, idx, w, l2, s2, None, *tail)
    again, _ = R.framed((rows, V), STORE[fmt], cuda, V + 2 * pad, shift=shift)
    l3 = torch.full((rows,), NAN, device=cuda)
    lrc.lrc_distill(z, t, idx, w, l3, None, again, *tail)
    assert torch.equal(l2, loss) and torch.equal(s2, lse) and torch.equal(l3, loss) and torch.equal(again, dz)
    # the gradient apart, with upstream gradients, one of them zero
    g = torch.rand(rows, device=cuda) + 0.5
    g[rows // 2] = 0
    part, partb = R.framed((rows, V), STORE[fmt], cuda, V + 2 * pad, shift=shift)
    lrc.lrc_distill_grad(z, t, idx, w, lse, g, part, *tail)
    _, _, want_dz, bdz = bounds(z, t, idx, w, tau, want, g, STORE[fmt])
    R.within(part, want_dz, bdz, "dz apart")
    R.frame_kept(part, partb)
    # without weights and upstream gradients
    lrc.lrc_distill_grad(z, t, idx, None, lse, None, part, *tail)
    ones = R.distill(z, t, idx, one, tau)
    _, _, want_dz, bdz = bounds(z, t, idx, one, tau, ones, one, STORE[fmt])
    R.within(part, want_dz, bdz, "dz without weights")


@pytest.mark.parametrize("rows,V,K", [(3, 700, 40), (2, 50001, 9), (1, 300001, 64), (200, 3000, 5)])
@pytest.mark.parametrize("fmt", ["f32", "bf16"])
def test_in_place(lrc, cuda, rows, V, K, fmt):
    z, _, t, idx, w = case(cuda, rows, V, K, fmt, "f32", 3)
    tail = (rows, V, K, V, K, V, 1.5, fmt, "f32")
    loss, lse, l2 = (torch.empty(rows, device=cuda) for _ in range(3))
    ref, z2 = torch.empty_like(z), z.clone()
    lrc.lrc_distill(z, t, idx, w, loss, lse, ref, *tail)
    lrc.lrc_distill(z2, t, idx, w, l2, None, z2, *tail)
    assert torch.equal(z2, ref) and torch.equal(l2, loss)
    z2 = z.clone()
    lrc.lrc_distill_grad(z2, t, idx, w, lse, None, z2, *tail)
    lrc.lrc_distill_grad(z, t, idx, w, lse, None, ref, *tail)
    assert torch.equal(z2, ref)


@pytest.mark.parametrize("fmt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("V", [50, 9000, 200001])
def test_rows_with_nothing_and_logits_that_are_not_finite(lrc, cuda, fmt, V):
    rows, K = 8, 4
    gen = torch.Generator(device=cuda).manual_seed(1)
    z = torch.randn((rows, V), generator=gen, device=cuda).to(STORE[fmt])
    t = torch.randn((rows, K), generator=gen, device=cuda)
    idx = torch.randint(0, V, (rows, K), generator=gen, device=cuda)
    w = torch.ones(rows, device=cuda)
    idx[0] = -1                       # no entries
    t[1] = -INF                       # no mass
    w[2] = 0                          # no weight, logits NaN
    z[2] = NAN
    z[3, V // 2] = NAN                # a NaN logit
    z[4] = -INF                       # only masked logits
    z[5, V - 1] = INF
    idx[6] = 0                        # a masked teacher place
    z[6, 0] = -INF
    idx[7] = 3                        # one place, four times
    loss, lse = torch.empty(rows, device=cuda), torch.empty(rows, device=cuda)
    dz = torch.empty_like(z)
    lrc.lrc_distill(z, t, idx, w, loss, lse, dz, rows, V, K, V, K, V, 1.0, fmt, "f32")
    assert bool((loss[:3] == 0).all()) and bool((dz[:3] == 0).all())
    assert bool(torch.isnan(loss[3:6]).all()) and bool(torch.isnan(dz[3:6]).any(1).all())
    assert float(lse[4]) == -INF and bool(torch.isfinite(lse[:2]).all()) and bool(torch.isnan(lse[[2, 3]]).all())
    assert float(loss[6]) == INF and bool(torch.isfinite(dz[6]).all())
    q = torch.softmax(z[6:8].double(), 1)
    assert abs(float(dz[6, 0]) + 1) <= OUT_U[STORE[fmt]] * 2
    assert abs(float(dz[7, 3]) - (float(q[1, 3]) - 1)) <= OUT_U[STORE[fmt]] * 2 + 1e-5
    part = torch.empty_like(z)
    lrc.lrc_distill_grad(z, t, idx, w, lse, None, part, rows, V, K, V, K, V, 1.0, fmt, "f32")
    assert bool((part[:3] == 0).all())


def test_gradient_against_differences(lrc, cuda):
    """Directional derivatives of the sum of the losses in binary64 (central
    differences, h = 1e-4: O(h^2) beside the gradient's binary32 error)."""
    rows, V, K, tau, h = 5, 200, 12, 1.7, 1e-4
    z, _, t, idx, w = case(cuda, rows, V, K, "f32", "f32", 9, holes=False)
    dz = torch.empty_like(z)
    lrc.lrc_distill(z, t, idx, w, None, None, dz, rows, V, K, V, K, V, tau, "f32", "f32")
    gen = torch.Generator(device=cuda).manual_seed(3)
    for _ in range(4):
        v = torch.randn(z.shape, generator=gen, device=cuda, dtype=torch.float64)
        diff = (R.distill(z.double() + h * v, t, idx, w, tau)[0].sum() -
                R.distill(z.double() - h * v, t, idx, w, tau)[0].sum()) / (2 * h)
        assert abs(float(diff) - float((dz.double() * v).sum())) <= 1e-4 * float((dz.double() * v).abs().sum())
    assert float(dz.double().sum(1).abs().max()) <= 1e-5 * tau * 1.5       # a row's gradient sums to zero


def test_teacher_rows_with_a_pitch(lrc, cuda):
    rows, V, K, ldt = 6, 900, 10, 13
    z, _, t, idx, w = case(cuda, rows, V, K, "bf16", "f16", 5)
    T, I = torch.full((rows, ldt), NAN, dtype=torch.float16, device=cuda), torch.zeros((rows, ldt), dtype=torch.int64, device=cuda)
    T[:, :K], I[:, :K] = t, idx
    out = []
    for tt, ii, ld in ((t, idx, K), (T, I, ldt)):
        loss, dz = torch.empty(rows, device=cuda), torch.empty_like(z)
        lrc.lrc_distill(z, tt, ii, w, loss, None, dz, rows, V, K, V, ld, V, 1.0, "bf16", "f16")
        out.append((loss, dz))
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])


def test_offsets_beyond_32_bits(lrc, cuda):
    """A pitch of 2^31 + 8 elements: the third row starts past 2^32."""
    rows, V, K, ld = 3, 5000, 20, 2 ** 31 + 8
    z0, _, t, idx, w = case(cuda, rows, V, K, "bf16", "f32", 4)
    w[:] = 1
    buf = torch.empty((rows - 1) * ld + V, dtype=torch.bfloat16, device=cuda)
    z = torch.as_strided(buf, (rows, V), (ld, 1))
    z.copy_(z0)
    loss, lse = torch.empty(rows, device=cuda), torch.empty(rows, device=cuda)
    lrc.lrc_distill(z, t, idx, w, loss, lse, z, rows, V, K, ld, K, ld, 1.0, "bf16", "f32")
    want = R.distill(z0, t, idx, w, 1.0)
    bloss, bl, want_dz, bdz = bounds(z0, t, idx, w, 1.0, want, torch.ones(rows, device=cuda), torch.bfloat16)
    R.within(loss, want[0], bloss)
    R.within(z, want_dz, bdz)


def test_no_rows_and_nothing_wanted(lrc, cuda):
    before = lrc.lrc_launch_count()
    lrc.lrc_distill(None, None, None, None, None, None, None, 0, 5, 2, 5, 2, 5, 1.0, "f32", "f32")
    z, _, t, idx, w = case(cuda, 2, 30, 3, "f32", "f32", 1)
    lrc.lrc_distill(z, t, idx, w, None, None, None, 2, 30, 3, 30, 3, 30, 1.0, "f32", "f32")
    assert lrc.lrc_launch_count() == before
