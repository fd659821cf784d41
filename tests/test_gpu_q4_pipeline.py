"""The 4-bit products of matrices that fill their pipelines: many blocks of columns
for every thread block, so that stages are filled again, barriers change phase and
accumulators are used block after block.  Against binary64 on sampled rows."""
import pytest
import torch

import layer_ref as R
from layer_ref import OUT, OUT_TINY, OUT_U, STORE, U

pytestmark = pytest.mark.gpu


def check(lrc, dev, m, n, b, group, zeros, fmt, sample=None):
    gen = torch.Generator(device=dev).manual_seed(m + n + b + group)
    dt, ot, G = STORE[fmt], OUT[fmt], -(-n // group)
    Q = torch.randint(0, 256, (m, lrc.lrc_q4_row_bytes(n)), generator=gen, device=dev, dtype=torch.uint8)
    s = (torch.rand((G, R.ld16(m)), generator=gen, device=dev) * 0.1 + 0.01).to(dt)
    z = torch.randint(0, 16, (G, R.ld16(m)), generator=gen, device=dev, dtype=torch.uint8) if zeros else None
    X = torch.full((b, R.ld16(n)), float("nan"), dtype=dt, device=dev)
    X[:, :n] = torch.randn((b, n), generator=gen, device=dev).to(dt)
    A = torch.randn((b, m), generator=gen, device=dev).to(ot)
    Y, buf = R.framed((b, m), ot, dev)
    lrc.lrc_q4_apply(Q, s, z, X, A, Y, m, n, b, group, fmt)
    R.frame_kept(Y, buf)
    assert bool(torch.isfinite(Y).all())
    rows = torch.arange(m, device=dev) if sample is None else \
        torch.unique(torch.cat([torch.randint(0, m, (sample,), generator=gen, device=dev),
                                torch.arange(8, device=dev), m - 1 - torch.arange(8, device=dev)]))
    v = R.q4_values(Q[rows], s[:, rows], None if z is None else z[:, rows], len(rows), n, group)
    x, a = X[:, :n].double(), A[:, rows].double()
    want = a + x @ v.t()
    # sums of a group, of the groups, and what is around them, each addition within 2 U
    # of its magnitude (the matrix instructions cut off)
    bound = 2 * U * (group + G + 40) * (x.abs() @ v.abs().t() + a.abs())
    R.within(Y[:, rows], want, bound + OUT_U[ot] * want.abs() * 1.01 + OUT_TINY[ot])
    again, _ = R.framed((b, m), ot, dev)
    lrc.lrc_q4_apply(Q, s, z, X, A, again, m, n, b, group, fmt)
    assert torch.equal(Y, again)


# on tcgen05: 128 blocks of columns, clusters of four at most
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("fmt,b", [("f16", 33), ("f16_o16", 64), ("bf16", 65), ("bf16", 50), ("f32", 11), ("f32", 22),
                                   ("f32", 43)])
def test_more_than_32_columns(lrc, cuda, group, zeros, fmt, b):
    check(lrc, cuda, 600, 16381, b, group, zeros, fmt)


# on mma.sync: rows for every multiprocessor, so that clusters are small, and blocks of
# columns for several turns of a ring of at most eight stages
@pytest.mark.parametrize("group,zeros", [(32, True), (64, False), (128, True)])
@pytest.mark.parametrize("fmt,b", [("f16", 1), ("bf16", 8), ("f16_o16", 13), ("bf16", 23), ("f16", 32), ("f32", 2),
                                   ("f32", 5), ("f32", 8), ("f32", 10)])
@pytest.mark.parametrize("m,n", [(16001, 16381), (5000, 8191), (700, 30011)])
def test_up_to_32_columns(lrc, cuda, group, zeros, fmt, b, m, n):
    check(lrc, cuda, m, n, b, group, zeros, fmt, sample=100)


# every multiprocessor has several tiles on tcgen05, one after the other
def test_more_tiles_than_multiprocessors(lrc, cuda):
    check(lrc, cuda, 60001, 2050, 70, 64, True, "f16", sample=200)


# the three parts of binary32 vectors fill their workspace more than once: at most 682
# vectors of 65536 entries a launch
@pytest.mark.parametrize("b", [682, 683, 1370])
def test_binary32_vectors_in_several_launches(lrc, cuda, b):
    check(lrc, cuda, 40, 65536, b, 128, False, "f32")
