"""Layer norm and its gradient on the GPU against binary64."""
import pytest
import torch

import layer_ref as R
from layer_ref import OUT, OUT_TINY, OUT_U, STORE, U

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1), (3, 2), (2, 31), (5, 33), (4, 256), (7, 1000), (64, 1138), (9, 4096), (3, 8191), (130, 512), (2, 16384),
          (1, 40001), (1, 100003)]


def sums(cols):
    """Error of a sum of cols terms spread over at least a warp's lanes, over
    the sum of the magnitudes, with room for the operations around it."""
    return (cols / 32 + 40) * U


def inputs(dev, rows, cols, fmt, pfmt, seed, ldx=None, shift=0):
    gen = torch.Generator(device=dev).manual_seed(seed)
    x, xb = R.framed((rows, cols), STORE[fmt], dev, ldx, shift=shift)
    x.copy_(torch.randn((rows, cols), generator=gen, device=dev) * 2 + 3)
    gamma = (1 + 0.3 * torch.randn(cols, generator=gen, device=dev)).to(STORE[pfmt]) if pfmt else None
    beta = torch.randn(cols, generator=gen, device=dev).to(STORE[pfmt]) if pfmt else None
    return x, gamma, beta, gen


def norm_bounds(x, gamma, beta, want, eps, out):
    """Bounds of y, mean and rstd: the mean is off by sums() of the mean
    magnitude, x - mu by that and a rounding, the variance by sums() and twice
    the mean's error (whose square is second order)."""
    y, mu, r = want
    cols = x.shape[1]
    k = sums(cols)
    x = x.double()
    g = torch.ones(cols, device=x.device, dtype=torch.float64) if gamma is None else gamma.double().abs()
    b = torch.zeros(cols, device=x.device, dtype=torch.float64) if beta is None else beta.double().abs()
    dmu = k * x.abs().mean(1, keepdim=True) + U * mu.abs()[:, None]
    xh = (x - mu[:, None]).abs() * r[:, None]
    dr = k + 2 * (dmu * r[:, None]) ** 2 + 2 * U * x.abs().amax(1, keepdim=True) * r[:, None]      # relative
    dy = g * r[:, None] * (dmu + U * (x - mu[:, None]).abs()) + g * xh * (dr + 4 * U) + 2 * U * (b + y.abs())
    return dy + OUT_U[out] * y.abs() + OUT_TINY[out], dmu[:, 0], (dr[:, 0] + 4 * U) * r


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("fmt,pfmt", [("f32", "f32"), ("f16", "f16"), ("f16_o16", "f32"), ("bf16", "bf16"), ("bf16", None)])
@pytest.mark.parametrize("pad,shift", [(0, 0), (5, 1)])
def test_norm(lrc, cuda, rows, cols, fmt, pfmt, pad, shift):
    x, gamma, beta, _ = inputs(cuda, rows, cols, fmt, pfmt, rows + cols, cols + pad, shift)
    y, yb = R.framed((rows, cols), OUT[fmt], cuda, cols + 2 * pad, shift=shift)
    mean, rstd = (torch.full((rows,), float("nan"), device=cuda) for _ in range(2))
    eps = 1e-5
    lrc.lrc_layer_norm(x, gamma, beta, y, mean, rstd, rows, cols, cols + pad, cols + 2 * pad, eps, fmt, pfmt or "f32")
    want = R.layer_norm(x, gamma, beta, eps)
    by, bm, br = norm_bounds(x, gamma, beta, want, eps, OUT[fmt])
    R.within(y, want[0], by, "y")
    R.within(mean, want[1], bm, "mean")
    R.within(rstd, want[2], br, "rstd")
    R.frame_kept(y, yb)


# Many rows, enough for blocks that keep going from row to row.
MANY = [(2432, 1025), (2500, 1100), (2433, 2048), (2440, 2050), (2600, 4104), (2437, 8192), (2435, 8190), (2441, 12296),
        (2433, 16384), (611, 513), (700, 1025), (609, 4097), (608, 9001), (608, 16383)]


@pytest.mark.parametrize("rows,cols", MANY)
@pytest.mark.parametrize("fmt,pfmt", [("f32", "f32"), ("f16", "f16"), ("f16_o16", "f32"), ("bf16", "bf16"), ("bf16", None)])
@pytest.mark.parametrize("pad,shift", [(0, 0), (5, 1)])
def test_norm_of_many_rows(lrc, cuda, rows, cols, fmt, pfmt, pad, shift):
    test_norm(lrc, cuda, rows, cols, fmt, pfmt, pad, shift)


@pytest.mark.parametrize("rows,cols,shift", [(2500, 4096, 0), (2500, 2050, 0), (700, 2049, 3)])
def test_many_rows_in_place_far_from_zero_and_not_finite(lrc, cuda, rows, cols, shift):
    x, gamma, beta, _ = inputs(cuda, rows, cols, "f32", "f32", 7, cols + shift, shift)
    x += 1e4
    x[5] = 3.0                                  # (equal values: x - mu is 0)
    y, mean, rstd = torch.empty(rows, cols, device=cuda), torch.empty(rows, device=cuda), torch.empty(rows, device=cuda)
    lrc.lrc_layer_norm(x, gamma, beta, y, mean, rstd, rows, cols, cols + shift, cols, 1e-5, "f32", "f32")
    want = R.layer_norm(x, gamma, beta, 1e-5)
    by, bm, br = norm_bounds(x, gamma, beta, want, 1e-5, torch.float32)
    keep = torch.arange(rows, device=cuda) != 5
    R.within(y[keep], want[0][keep], by[keep], "y")
    R.within(mean, want[1], bm, "mean")
    R.within(rstd[keep], want[2][keep], br[keep], "rstd")
    assert torch.equal(y[5], beta.float()) and mean[5].item() == 3.0
    x[9, 2], x[11, cols - 1] = float("nan"), float("inf")
    lrc.lrc_layer_norm(x, gamma, beta, x, None, None, rows, cols, cols + shift, cols + shift, 1e-5, "f32", "f32")
    bad = torch.zeros(rows, dtype=torch.bool, device=cuda)
    bad[9] = bad[11] = True
    assert x[bad].isnan().all() and torch.equal(x[~bad], y[~bad])
    x[3] = 2.0
    lrc.lrc_layer_norm(x, gamma, beta, x, None, rstd, rows, cols, cols + shift, cols + shift, 0.0, "f32", "f32")
    assert x[3].isnan().all() and rstd[3].item() == float("inf")


def test_norm_of_rows_far_from_zero(lrc, cuda):
    """A mean 10^4 standard deviations away: the squares are of x - mu."""
    rows, cols = 6, 3000
    gen = torch.Generator(device=cuda).manual_seed(1)
    x = 1e4 + torch.randn((rows, cols), generator=gen, device=cuda)
    y = torch.empty_like(x)
    mean, rstd = torch.empty(rows, device=cuda), torch.empty(rows, device=cuda)
    lrc.lrc_layer_norm(x, None, None, y, mean, rstd, rows, cols, cols, cols, 0.0, "f32", "f32")
    want = R.layer_norm(x, None, None, 0.0)
    by, bm, br = norm_bounds(x, None, None, want, 0.0, torch.float32)
    R.within(y, want[0], by)
    R.within(rstd, want[2], br)


def test_norm_in_place_and_without_statistics(lrc, cuda):
    for cols in (100, 1024, 30001, 70000):
        x, gamma, beta, _ = inputs(cuda, 4, cols, "bf16", "f32", 3)
        ref = torch.empty_like(x)
        lrc.lrc_layer_norm(x, gamma, beta, ref, None, None, 4, cols, cols, cols, 1e-6, "bf16", "f32")
        lrc.lrc_layer_norm(x, gamma, beta, x, None, None, 4, cols, cols, cols, 1e-6, "bf16", "f32")
        assert torch.equal(x, ref)


def test_norm_of_rows_that_are_not_finite_or_constant(lrc, cuda):
    rows, cols = 5, 200
    x = torch.randn((rows, cols), device=cuda)
    x[1, 7] = float("nan")
    x[2, 9] = float("inf")
    x[3] = 2.5
    y = torch.empty_like(x)
    mean, rstd = torch.empty(rows, device=cuda), torch.empty(rows, device=cuda)
    lrc.lrc_layer_norm(x, None, None, y, mean, rstd, rows, cols, cols, cols, 1e-5, "f32", "f32")
    assert bool(torch.isnan(y[1:3]).all()) and bool(torch.isfinite(y[[0, 3, 4]]).all())
    assert bool((y[3] == 0).all())
    lrc.lrc_layer_norm(x, None, None, y, mean, rstd, rows, cols, cols, cols, 0.0, "f32", "f32")
    assert bool(torch.isnan(y[3]).all()) and bool(torch.isinf(rstd[3]))


def grad_bounds(dy, x, gamma, mu, r, want, out):
    dx = want[0]
    rows, cols = x.shape
    k = sums(cols)
    r = r.double()[:, None]
    xc = x.double() - mu.double()[:, None]
    xh = xc.abs() * r
    d = dy.double().abs() * (1 if gamma is None else gamma.double().abs())
    bx = r * (4 * U * d + (k + 4 * U) * d.mean(1, keepdim=True) + (2 * k + 8 * U) * xh * (d * xh).mean(1, keepdim=True))
    kr = (rows + 40) * U
    return (bx + OUT_U[out] * dx.abs() + OUT_TINY[out], kr * (dy.double().abs() * xh).sum(0),
            kr * dy.double().abs().sum(0))


@pytest.mark.parametrize("rows,cols", SHAPES + [(700, 129), (1025, 64), (1300, 9000), (700, 20001), (1901, 4097)])
@pytest.mark.parametrize("fmt,pfmt", [("f32", "f32"), ("f16", "f16"), ("f16_o16", "f16"), ("bf16", "f32"), ("bf16", None)])
@pytest.mark.parametrize("pad,shift", [(0, 0), (3, 1)])
def test_grad(lrc, cuda, rows, cols, fmt, pfmt, pad, shift):
    x, gamma, _, gen = inputs(cuda, rows, cols, fmt, pfmt, rows + cols, cols + pad, shift)
    dy, _ = R.framed((rows, cols), OUT[fmt], cuda, cols + 2 * pad, shift=shift)
    dy.copy_(torch.randn((rows, cols), generator=gen, device=cuda) + 0.2)
    _, mu, r = R.layer_norm(x, None, None, 1e-5)
    mu, r = mu.float(), r.float()
    dx, dxb = R.framed((rows, cols), STORE[fmt], cuda, cols + pad, shift=shift)
    dg, db = (torch.full((cols,), float("nan"), device=cuda) for _ in range(2))
    args = (rows, cols, cols + 2 * pad, cols + pad, cols + pad, fmt, pfmt or "f32")
    lrc.lrc_layer_norm_grad(dy, x, gamma, mu, r, dx, dg, db, *args)
    want = R.layer_norm_grad(dy, x, gamma, mu, r)
    bx, bg, bb = grad_bounds(dy, x, gamma, mu, r, want, STORE[fmt])
    R.within(dx, want[0], bx, "dx")
    R.within(dg, want[1], bg, "dgamma")
    R.within(db, want[2], bb, "dbeta")
    R.frame_kept(dx, dxb)
    # each output alone, and twice: the same bits
    for keep in ("x", "g", "b", "xgb"):
        o = [torch.full_like(t, float("nan")) if c in keep else None for t, c in ((dg, "g"), (db, "b"))]
        ox, _ = R.framed((rows, cols), STORE[fmt], cuda, cols + pad, shift=shift)
        lrc.lrc_layer_norm_grad(dy, x, gamma, mu, r, ox if "x" in keep else None, *o, *args)
        assert "x" not in keep or torch.equal(ox, dx)
        assert all(t is None or torch.equal(t, ref) for t, ref in zip(o, (dg, db)))
    if fmt == "f32" and not pad:                   # over its own inputs
        for alias in (dy, x):
            a = alias.clone()
            ins = (a, x) if alias is dy else (dy, a)
            lrc.lrc_layer_norm_grad(*ins, gamma, mu, r, a, dg, db, *args)
            assert torch.equal(a, dx)


def test_grad_against_differences(lrc, cuda):
    """Directional derivatives of a weighted sum of outputs, in binary64: the
    central difference is off by O(h^2) of the third derivative (h = 1e-4: far
    below the gradient's own binary32 error, 1e-4 here with room)."""
    rows, cols, eps, h = 4, 96, 1e-5, 1e-4
    gen = torch.Generator(device=cuda).manual_seed(11)
    x, gamma, beta, dy = (torch.randn(s, generator=gen, device=cuda) for s in ((rows, cols), (cols,), (cols,), (rows, cols)))
    y, mu, r = torch.empty_like(x), torch.empty(rows, device=cuda), torch.empty(rows, device=cuda)
    lrc.lrc_layer_norm(x, gamma, beta, y, mu, r, rows, cols, cols, cols, eps, "f32", "f32")
    dx, dg, db = torch.empty_like(x), torch.empty(cols, device=cuda), torch.empty(cols, device=cuda)
    lrc.lrc_layer_norm_grad(dy, x, gamma, mu, r, dx, dg, db, rows, cols, cols, cols, cols, "f32", "f32")

    def f(x, gamma, beta):
        return float((R.layer_norm(x, gamma, beta, eps)[0] * dy.double()).sum())

    at = [t.double() for t in (x, gamma, beta)]
    for i, grad in enumerate((dx, dg, db)):
        for _ in range(4):
            v = torch.randn(at[i].shape, generator=gen, device=cuda, dtype=torch.float64)
            up, down = list(at), list(at)
            up[i], down[i] = at[i] + h * v, at[i] - h * v
            diff = (f(*up) - f(*down)) / (2 * h)
            assert abs(diff - float((grad.double() * v).sum())) <= 1e-4 * float((grad.double() * v).abs().sum())


def test_no_rows(lrc, cuda):
    dg, db = (torch.full((70,), float("nan"), device=cuda) for _ in range(2))
    lrc.lrc_layer_norm_grad(None, None, None, None, None, None, dg, db, 0, 70, 70, 70, 70, "f32", "f32")
    assert bool((dg == 0).all()) and bool((db == 0).all())
    before = lrc.lrc_launch_count()
    lrc.lrc_layer_norm(None, None, None, None, None, None, 0, 70, 70, 70, 1e-5, "f32", "f32")
    lrc.lrc_layer_norm_grad(None, None, None, None, None, None, None, None, 0, 70, 70, 70, 70, "f32", "f32")
    assert lrc.lrc_launch_count() == before


def test_offsets_beyond_32_bits(lrc, cuda):
    """A pitch of 2^31 + 8 elements: the third row starts past 2^32."""
    rows, cols, ld = 3, 500, 2 ** 31 + 8
    buf = torch.empty((rows - 1) * ld + cols, dtype=torch.bfloat16, device=cuda)
    x = torch.as_strided(buf, (rows, cols), (ld, 1))
    x.copy_(torch.randn((rows, cols), device=cuda))
    y = torch.empty((rows, cols), dtype=torch.bfloat16, device=cuda)
    mean, rstd = torch.empty(rows, device=cuda), torch.empty(rows, device=cuda)
    lrc.lrc_layer_norm(x, None, None, y, mean, rstd, rows, cols, ld, cols, 1e-5, "bf16", "f32")
    want = R.layer_norm(x, None, None, 1e-5)
    R.within(y, want[0], norm_bounds(x, None, None, want, 1e-5, torch.bfloat16)[0])
    dx = torch.as_strided(torch.empty_like(buf), (rows, cols), (ld, 1))
    dg, db = torch.empty(cols, device=cuda), torch.empty(cols, device=cuda)
    lrc.lrc_layer_norm_grad(y, x, None, mean, rstd, dx, dg, db, rows, cols, cols, ld, ld, "bf16", "f32")
    want = R.layer_norm_grad(y, x, None, mean, rstd)
    bx, bg, _ = grad_bounds(y, x, None, mean, rstd, want, torch.bfloat16)
    R.within(dx, want[0], bx)
    R.within(dg, want[1], bg)


def test_on_another_stream(lrc, cuda):
    """The partial sums live in a workspace per stream."""
    rows, cols = 300, 700
    x, gamma, _, gen = inputs(cuda, rows, cols, "f32", "f32", 2)
    dy = torch.randn((rows, cols), generator=gen, device=cuda)
    mu, r = (t.float() for t in R.layer_norm(x, None, None, 1e-5)[1:])
    tail = (rows, cols, cols, cols, cols, "f32", "f32")
    ref = [torch.empty_like(dy), torch.empty(cols, device=cuda), torch.empty(cols, device=cuda)]
    lrc.lrc_layer_norm_grad(dy, x, gamma, mu, r, *ref, *tail)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for i in range(8):
        o = [torch.full_like(t, float("nan")) for t in ref]
        streams[i % 2].wait_stream(torch.cuda.current_stream())
        lrc.lrc_layer_norm_grad(dy, x, gamma, mu, r, *o, *tail, stream=streams[i % 2])
        outs.append(o)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for o in outs for a, b in zip(o, ref))
