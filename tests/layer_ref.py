"""Plain binary64 forms of the operators around a compressed layer, on torch
tensors, and what their tests share.  Error bounds: U is the unit roundoff of
binary32, OUT_U of the output types."""
import math

import torch

U = 2.0 ** -24
STORE = {"f32": torch.float32, "f16": torch.float16, "f16_o16": torch.float16, "bf16": torch.bfloat16,
         "f32tc": torch.float32, "f64": torch.float64}
OUT = {"f32": torch.float32, "f16": torch.float32, "f16_o16": torch.float16, "bf16": torch.bfloat16,
       "f32tc": torch.float32}
OUT_U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
# half the spacing of the smallest numbers
OUT_TINY = {torch.float32: 2.0 ** -150, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}

NIBBLE = [0, 4, 1, 5, 2, 6, 3, 7]        # 4-bit place of column e of a word


def ld16(cols):
    return (cols + 15) // 16 * 16


def q4_unpack(Q, n):
    """Codes of a laid-out matrix (m x row bytes, uint8) as int64, m x n."""
    m = Q.shape[0]
    c = torch.arange(n, device=Q.device)
    j, t, e = c % 128 // 32, c % 32 // 8, c % 8
    nib = torch.tensor(NIBBLE, device=Q.device)[e]
    byte = c // 128 * 64 + (4 * t + j) * 4 + nib // 2
    return (Q[:, byte].long() >> (4 * (nib % 2))) & 15


def q4_pack(codes):
    """The inverse: codes m x n to m x row bytes (pad columns get code 8)."""
    m, n = codes.shape
    nb = -(-n // 128) * 128
    full = torch.full((m, nb), 8, dtype=torch.int64, device=codes.device)
    full[:, :n] = codes
    c = torch.arange(nb, device=codes.device)
    j, t, e = c % 128 // 32, c % 32 // 8, c % 8
    nib = torch.tensor(NIBBLE, device=codes.device)[e]
    byte = c // 128 * 64 + (4 * t + j) * 4 + nib // 2
    Q = torch.zeros((m, nb // 2), dtype=torch.int64, device=codes.device)
    Q.index_add_(1, byte, full << (4 * (nib % 2)))
    return Q.to(torch.uint8)


def spread(a, m, n, group):
    """Group values (groups x >= m) over the columns of their groups, m x n, binary64."""
    return a[:, :m].double().t().repeat_interleave(group, 1)[:, :n]


def q4_values(Q, scales, zeros, m, n, group):
    z = 8.0 if zeros is None else spread(zeros, m, n, group)
    return (q4_unpack(Q, n).double() - z) * spread(scales, m, n, group)


def layer_norm(x, gamma, beta, eps):
    """(y, mean, rstd) in binary64."""
    x = x.double()
    mu = x.mean(1, keepdim=True)
    r = 1 / torch.sqrt(((x - mu) ** 2).mean(1, keepdim=True) + eps)
    y = (x - mu) * r
    if gamma is not None:
        y = y * gamma.double()
    if beta is not None:
        y = y + beta.double()
    return y, mu[:, 0], r[:, 0]


def layer_norm_grad(dy, x, gamma, mu, r):
    """(dx, dgamma, dbeta) in binary64 for given mean and rstd."""
    dy, r = dy.double(), r.double()[:, None]
    xh = (x.double() - mu.double()[:, None]) * r
    d = dy if gamma is None else dy * gamma.double()
    dx = r * (d - d.mean(1, keepdim=True) - xh * (d * xh).mean(1, keepdim=True))
    return dx, (dy * xh).sum(0), dy.sum(0)


def distill(z, t, idx, w, tau):
    """(loss, lse, dz, p at the teacher's entries) in binary64; w of length rows."""
    rows, V = z.shape
    z = z.double() / tau
    lse = torch.logsumexp(z, 1)
    loss = torch.zeros(rows, dtype=torch.float64, device=z.device)
    dz = torch.zeros_like(z)
    ps = torch.zeros(t.shape, dtype=torch.float64, device=z.device)
    for r in range(rows):
        here = [k for k in range(t.shape[1]) if 0 <= int(idx[r, k]) < V and float(t[r, k]) != -math.inf]
        if not here or float(w[r]) == 0.0:
            continue
        tr = t[r, here].double() / tau
        logp = tr - torch.logsumexp(tr, 0)
        p, i = torch.exp(logp), idx[r, here].long()
        ps[r, here] = p
        loss[r] = tau ** 2 * float(w[r]) * (p * (logp - (z[r, i] - lse[r]))).sum()
        dz[r] = torch.exp(z[r] - lse[r]).index_add_(0, i, -p) * (tau * float(w[r]))
    return loss, lse, dz, ps


def within(got, want, bound, what=""):
    """|got - want| <= bound, entry by entry; NaN and infinities in the same places."""
    got, want = got.double(), want.double()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isfinite(got), fine), what
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    assert bool((same | fine).all()), what
    off = torch.where(fine, (got - want).abs() - bound, torch.zeros_like(want))
    worst = float(off.max()) if off.numel() else 0.0
    assert worst <= 0, (what, worst, int(off.argmax()))


def framed(shape, dtype, dev, ld=None, fill=float("nan"), shift=0):
    """A rows x cols view (row pitch ld, `shift` elements into its buffer) whose
    surroundings hold `fill`, and the buffer."""
    rows, cols = shape
    ld = cols if ld is None else ld
    buf = torch.full((shift + rows * ld + 64,), fill, dtype=dtype, device=dev)
    return buf[shift:shift + rows * ld].view(rows, ld)[:, :cols], buf


def frame_kept(view, buf):
    """Nothing around the view was written (the frame is NaN)."""
    b = buf.clone()
    rows, cols = view.shape
    b[view.storage_offset():view.storage_offset() + rows * view.stride(0)].view(rows, -1)[:, :cols] = float("nan")
    assert bool(torch.isnan(b).all())
