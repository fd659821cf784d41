"""Distillation where every thread block has several rows, one after the other:
teacher entries prepared ahead, elements outside the whole 16 bytes loaded a row
ahead, a ring that goes on from row to row.  Against binary64, every row."""
import math

import pytest
import torch

import layer_ref as R
from layer_ref import OUT_TINY, OUT_U, STORE, U

pytestmark = pytest.mark.gpu


def reference(z, t, idx, w, tau):
    """(loss, lse, dz, p) in binary64, as layer_ref.distill, all rows at once."""
    V = z.shape[1]
    zz = z.double() / tau
    lse = torch.logsumexp(zz, 1)
    there = (idx >= 0) & (idx < V) & (t != -math.inf)
    tt = torch.where(there, t.double() / tau, -math.inf)
    on = there.any(1) & (w != 0)
    logp = torch.where(there & on[:, None], tt - torch.logsumexp(tt, 1, keepdim=True), -math.inf)
    p = torch.exp(logp)
    at = idx.clamp(0, V - 1)
    kl = torch.where(p > 0, p * (logp - (zz.gather(1, at) - lse[:, None])), 0.0).sum(1)
    loss = torch.where(on, tau ** 2 * w.double() * kl, 0.0)
    dz = torch.exp(zz - lse[:, None]).scatter_add_(1, at, -p) * (tau * w.double())[:, None]
    return loss, lse, torch.where(on[:, None], dz, 0.0), p


def case(dev, rows, V, K, fmt, tfmt, pad, shift, seed):
    gen = torch.Generator(device=dev).manual_seed(seed)
    z, buf = R.framed((rows, V), STORE[fmt], dev, V + pad, shift=shift)
    for r in range(0, rows, 64):
        z[r:r + 64] = torch.randn((min(64, rows - r), V), generator=gen, device=dev) * 2
    z[:, 5::97] = -math.inf
    t = (torch.randn((rows, K), generator=gen, device=dev) * 2).to(STORE[tfmt])
    idx = torch.randint(0, V, (rows, K), generator=gen, device=dev)
    idx[idx % 97 == 5] = 1
    idx[torch.rand((rows, K), generator=gen, device=dev) < 0.2] = -1
    t[torch.rand((rows, K), generator=gen, device=dev) < 0.1] = -math.inf
    w = torch.rand(rows, generator=gen, device=dev) + 0.5
    w[3::7] = 0                                          # rows without weight and without
    idx[5::11] = V                                       # entries between the others
    return z, buf, t, idx, w


SHAPES = [(2500, 640, 9, 0, 0), (2500, 641, 1024, 3, 1), (1500, 7001, 33, 0, 3),        # four blocks a multiprocessor
          (1000, 20001, 300, 1, 2), (1000, 20000, 7, 0, 0),                              # two
          (500, 70001, 40, 2, 1), (500, 40000, 5, 8, 0), (333, 40004, 1024, 1, 0),       # one; kept, or in 32 bits read twice
          (400, 131072, 50, 0, 0), (330, 150001, 20, 0, 5)]


@pytest.mark.parametrize("rows,V,K,pad,shift", SHAPES)
@pytest.mark.parametrize("fmt,tfmt,tau", [("f32", "f16", 1.0), ("bf16", "f32", 2.0), ("f16", "bf16", 0.5)])
def test_several_rows_a_block(lrc, cuda, rows, V, K, pad, shift, fmt, tfmt, tau):
    z, zb, t, idx, w = case(cuda, rows, V, K, fmt, tfmt, pad, shift, rows + V)
    loss, lse, dz, p = reference(z, t, idx, w, tau)
    # a sum over at least 128 partial sums; exponents rounded at the size of z / tau
    zf = torch.where(torch.isfinite(z), z, torch.zeros_like(z)).double().abs().amax(1) / tau + lse.abs()
    tf = torch.where(torch.isfinite(t), t, torch.zeros_like(t)).double().abs().amax(1) / tau
    bl, bt = (V / 128 + 40 + 8 * zf) * U, (K / 32 + 40 + 8 * tf) * U
    b_loss = tau ** 2 * w.double() * (2 * bl + bt * (2 + 2 * tf + 2 * zf)) + 2 * U * loss.abs()
    at = idx.clamp(0, V - 1)

    def b_dz(dz, g):
        c = (tau * w.double() * g.double())[:, None]
        b = torch.exp(z.double() / tau - lse[:, None]) * (2 * bl[:, None] + 8 * U)
        b.scatter_add_(1, at, p * (2 * bt[:, None] + 8 * U))
        return b.mul_(c).add_(OUT_TINY[STORE[fmt]]).add_(dz.abs(), alpha=OUT_U[STORE[fmt]] * 1.01)

    for other in (pad, pad + 1):                         # results that start where the logits do, and elsewhere
        tail = (rows, V, K, V + pad, K, V + other, tau, fmt, tfmt)
        got, buf = R.framed((rows, V), STORE[fmt], cuda, V + other, shift=shift)
        lo, ls = torch.full((rows,), math.nan, device=cuda), torch.full((rows,), math.nan, device=cuda)
        lrc.lrc_distill(z, t, idx, w, lo, ls, got, *tail)
        R.within(ls, lse, bl, "lse")
        R.within(lo, loss, b_loss, "loss")
        R.within(got, dz, b_dz(dz, torch.ones_like(w)), "dz")
        R.frame_kept(got, buf)
        again = torch.full((rows,), math.nan, device=cuda)
        lrc.lrc_distill(z, t, idx, w, again, None, None, *tail)
        assert torch.equal(again, lo)
        g = torch.rand(rows, device=cuda) + 0.5
        g[::13] = 0
        apart, buf = R.framed((rows, V), STORE[fmt], cuda, V + other, shift=shift)
        lrc.lrc_distill_grad(z, t, idx, w, ls, g, apart, *tail)
        R.within(apart, dz * g.double()[:, None], b_dz(dz * g.double()[:, None], g), "dz apart")
        R.frame_kept(apart, buf)
        if other == pad:                                 # in place, later rows' copies and teacher entries on their way
            z2 = zb.clone()[shift:shift + rows * (V + pad)].view(rows, V + pad)[:, :V]
            lrc.lrc_distill(z2, t, idx, w, lo, None, z2, *tail)
            assert torch.equal(z2, got)
            z2.copy_(z)
            lrc.lrc_distill_grad(z2, t, idx, w, ls, g, z2, *tail)
            assert torch.equal(z2, apart)
