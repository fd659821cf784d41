"""4-bit matrices on the GPU: rounding (bit for bit), widening, and the product
with vectors against binary64."""
import numpy as np
import pytest
import torch

import layer_ref as R
from layer_ref import OUT, OUT_TINY, OUT_U, STORE, U

pytestmark = pytest.mark.gpu


def rounded_by_definition(W, group, zeros, dt):
    """Codes, scales and zeros by the stated binary32 steps, in numpy."""
    W = W.detach().float().cpu().numpy()
    m, n = W.shape
    f32, G = np.float32, -(-n // group)
    w = np.zeros((m, G * group), f32)
    w[:, :n] = W
    w = w.reshape(m, G, group)
    bad = ~np.isfinite(w).all(2)
    v = np.where(np.isfinite(w), w, f32(0))
    lo, hi = np.minimum(v.min(2), f32(0)), np.maximum(v.max(2), f32(0))
    with np.errstate(over="ignore"):
        s = (hi - lo) * f32(1 / 15) if zeros else np.maximum(hi, -lo) * f32(1 / 7)
    s = np.minimum(s, f32(torch.finfo(dt).max))
    s = torch.from_numpy(s).to(dt).float().numpy()
    none = s < f32(2.0 ** -126)
    s = np.where(none, f32(0), s)
    inv = np.where(none, f32(0), f32(1) / np.where(none, f32(1), s)).astype(f32)
    z = np.clip(np.rint(-lo * inv), 0, 15) if zeros else np.full(s.shape, f32(8))
    q = np.clip(np.rint(v * inv[..., None]) + z[..., None], 0, 15)
    q[bad], z[bad], s[bad] = 8, 8, np.nan
    return q.reshape(m, -1)[:, :n].astype(np.int64), s.T, z.T.astype(np.int64)


@pytest.mark.parametrize("m,n", [(1, 1), (3, 127), (17, 128), (5, 129), (64, 512), (33, 1000), (7, 31)])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("src,fmt", [("f32", "f16"), ("bf16", "bf16"), ("f16", "f32"), ("f64", "f16_o16")])
def test_round_follows_the_definition(lrc, cuda, m, n, group, zeros, src, fmt):
    gen = torch.Generator(device=cuda).manual_seed(m * n + group)
    W = (torch.randn((m, n), generator=gen, device=cuda) * 0.05).to(STORE[src])
    q = lrc.q4_matrix(W, fmt, group, zeros)
    codes, s, z = rounded_by_definition(W, group, zeros, STORE[fmt])
    assert np.array_equal(R.q4_unpack(q.Q, n).cpu().numpy(), codes)
    assert np.array_equal(q.scales[:, :m].float().cpu().numpy(), s)
    if zeros:
        assert np.array_equal(q.zeros[:, :m].cpu().numpy(), z)
    pad = R.q4_unpack(q.Q, q.Q.shape[1] * 2)[:, n:]          # pad columns stand for zero
    zz = 8 if q.zeros is None else q.zeros[-1, :m].long()[:, None]
    last = pad[:, :(-n) % group]
    assert bool((last == zz).all())


@pytest.mark.parametrize("zeros", [False, True])
def test_round_at_the_ends_of_the_ranges(lrc, cuda, zeros):
    """Zeros, subnormals, the largest numbers (a binary16 scale saturates),
    one-signed groups, ties, infinities and NaN: each in a group of its own."""
    group, inf, nan = 32, float("inf"), float("nan")
    rows = [[0.0] * 32, [1e-45] * 32, [2.0 ** -127] + [0.0] * 31, [3.4e38, -3.4e38] * 16, [1e6] * 32, [-1e6] * 32,
            [0.5 * k for k in range(-16, 16)], [0.25] * 31 + [7.0], [inf] + [1.0] * 31, [1.0] * 31 + [nan],
            [-inf, inf] + [0.0] * 30, [-0.0] * 32, [1e-7] * 32, [6e-8, -3e-8] * 16]
    W = torch.tensor(rows, dtype=torch.float32, device=cuda)
    for fmt in ("f32", "f16", "bf16"):
        q = lrc.q4_matrix(W, fmt, group, zeros)
        codes, s, z = rounded_by_definition(W, group, zeros, STORE[fmt])
        m = W.shape[0]
        assert np.array_equal(R.q4_unpack(q.Q, 32).cpu().numpy(), codes), fmt
        assert np.array_equal(q.scales[:, :m].float().cpu().numpy(), s, equal_nan=True), fmt
        if zeros:
            assert np.array_equal(q.zeros[:, :m].cpu().numpy(), z), fmt


@pytest.mark.parametrize("src", ["f16", "bf16"])
@pytest.mark.parametrize("n", [24, 39, 130, 517, 1040])
@pytest.mark.parametrize("pad", [0, 1, 6, 8])
def test_round_of_16_bit_rows_that_start_anywhere(lrc, cuda, src, n, pad):
    """Every place within 16 bytes; a NaN beside a row would show; the ends of
    the ranges in groups of their own."""
    inf, nan, m = float("inf"), float("nan"), 41
    gen = torch.Generator(device=cuda).manual_seed(n + pad)
    for shift in range(9):
        W, _ = R.framed((m, n), STORE[src], cuda, n + pad, shift=shift)
        W.copy_(torch.randn((m, n), generator=gen, device=cuda) * 0.05)
        W[3] = 0.0
        W[4] = -W[4].abs()
        W[5] = W[5].abs()
        W[6, n // 2], W[7, 0], W[8, n - 1], W[9, n // 3] = nan, inf, -inf, -nan
        W[10] *= 2.0 ** -18                                   # binary16: subnormal
        W[11, ::2], W[11, 1::2] = 6e4, -6e4
        W[12] = -0.0
        for group, zeros, fmt in ((32, True, "f32"), (64, False, "bf16"), (128, True, "f16")):
            Q = torch.empty((m, lrc.lrc_q4_row_bytes(n)), dtype=torch.uint8, device=cuda)
            ld, groups = lrc.lrc_packed_ld(m), -(-n // group)
            scales = torch.empty((groups, ld), dtype=STORE[fmt], device=cuda)
            zc = torch.empty((groups, ld), dtype=torch.uint8, device=cuda) if zeros else None
            lrc.lrc_q4_round(W, src, m, n, n + pad, Q, scales, zc, group, fmt)
            codes, s, z = rounded_by_definition(W, group, zeros, STORE[fmt])
            assert np.array_equal(R.q4_unpack(Q, n).cpu().numpy(), codes)
            assert np.array_equal(scales[:, :m].float().cpu().numpy(), s, equal_nan=True)
            if zeros:
                assert np.array_equal(zc[:, :m].cpu().numpy(), z)


@pytest.mark.parametrize("m,n,ld", [(1, 1, 1), (9, 130, 131), (64, 512, 512), (31, 1001, 1001), (8, 257, 272)])
@pytest.mark.parametrize("group,zeros", [(32, True), (64, False), (128, True)])
@pytest.mark.parametrize("fmt,dfmt", [("f16", "f64"), ("bf16", "f32"), ("f32", "f32"), ("f16", "bf16"), ("bf16", "f16"),
                                      ("f32", "f64")])
def test_widen(lrc, cuda, m, n, ld, group, zeros, fmt, dfmt):
    gen = torch.Generator(device=cuda).manual_seed(n)
    q = lrc.q4_matrix(torch.randn((m, n), generator=gen, device=cuda), fmt, group, zeros)
    dst, buf = R.framed((m, n), STORE[dfmt], cuda, ld)
    lrc.lrc_q4_widen(q.Q, q.scales, q.zeros, group, fmt, m, n, dst, dfmt, ld)
    want = R.q4_values(q.Q, q.scales, q.zeros, m, n, group)       # exact: at most 28 bits
    if dfmt != "f64":
        want = want.float().to(STORE[dfmt])
    assert torch.equal(dst, want)
    R.frame_kept(dst, buf)


def random_q4(dev, m, n, group, zeros, fmt, seed, poison=True):
    """A random matrix in the layout, with whatever in the pad columns."""
    gen = torch.Generator(device=dev).manual_seed(seed)
    nb = -(-n // 128) * 128
    Q = R.q4_pack(torch.randint(0, 16, (m, nb if poison else n), generator=gen, device=dev))
    G, ldm = -(-n // group), R.ld16(m)
    s = torch.full((G, ldm), float("nan"), dtype=STORE[fmt], device=dev)
    s[:, :m] = (torch.rand((G, m), generator=gen, device=dev) * 0.1 + 0.01).to(STORE[fmt])
    z = torch.randint(0, 16, (G, ldm), generator=gen, device=dev).to(torch.uint8) if zeros else None
    return Q, s, z


def apply_bound(values, X, A, n, group, out):
    """Sums of at most `group` exact products, then of the groups, each addition
    within 2 U of its result's magnitude (the tensor cores truncate), one
    scaling and one addition of A, one rounding of the output."""
    S = X.abs() @ values.abs().t() + (0 if A is None else A.double().abs())
    want = X @ values.t() + (0 if A is None else A.double())
    terms = group + -(-n // group) + 40
    return want, 2 * U * terms * S + OUT_U[out] * want.abs() * 1.01 + OUT_TINY[out]


@pytest.mark.parametrize("fmt", ["f32", "f16", "f16_o16", "bf16", "f32tc"])
@pytest.mark.parametrize("m,n,b", [(1, 1, 1), (5, 31, 3), (16, 128, 1), (17, 129, 2), (100, 1000, 5), (512, 512, 1),
                                   (33, 4099, 8), (257, 640, 9), (64, 16381, 1), (130, 257, 33), (48, 384, 64),
                                   (16, 144, 65), (31, 130, 200), (1, 5000, 1), (2048, 96, 7)])
@pytest.mark.parametrize("group,zeros,add", [(32, False, False), (64, True, True), (128, False, True), (128, True, False)])
def test_apply(lrc, cuda, fmt, m, n, b, group, zeros, add):
    dt, ot = STORE[fmt], OUT[fmt]
    Q, s, z = random_q4(cuda, m, n, group, zeros, fmt, m + n + b)
    gen = torch.Generator(device=cuda).manual_seed(7)
    X = torch.full((b, R.ld16(n)), float("nan"), dtype=dt, device=cuda)        # pads are not read
    X[:, :n] = torch.randn((b, n), generator=gen, device=cuda).to(dt)
    A = torch.randn((b, m), generator=gen, device=cuda).to(ot) if add else None
    Y, buf = R.framed((b, m), ot, cuda)
    lrc.lrc_q4_apply(Q, s, z, X, A, Y, m, n, b, group, fmt)
    want, bound = apply_bound(R.q4_values(Q, s, z, m, n, group), X[:, :n].double(), A, n, group, ot)
    R.within(Y, want, bound)
    R.frame_kept(Y, buf)
    again, _ = R.framed((b, m), ot, cuda)
    lrc.lrc_q4_apply(Q, s, z, X, A, again, m, n, b, group, fmt)
    assert torch.equal(Y, again)                                               # deterministic
    if add:                                                                    # in place
        lrc.lrc_q4_apply(Q, s, z, X, A, A, m, n, b, group, fmt)
        assert torch.equal(A, Y)


@pytest.mark.parametrize("fmt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("b", [1, 6, 40])
def test_apply_keeps_what_is_not_finite_in_its_rows(lrc, cuda, fmt, b):
    """A NaN scale shows in its matrix row alone, an infinite entry of X in its
    vector alone; the rest is as without."""
    m, n, group = 70, 300, 64
    dt, ot = STORE[fmt], OUT[fmt]
    Q, s, z = random_q4(cuda, m, n, group, False, fmt, 5)
    X = torch.zeros((b, R.ld16(n)), dtype=dt, device=cuda)
    X[:, :n] = torch.randn((b, n), generator=torch.Generator(device=cuda).manual_seed(1), device=cuda).to(dt)
    s[1, 9] = float("nan")
    X[b - 1, 77] = float("inf")
    Y = torch.empty((b, m), dtype=ot, device=cuda)
    lrc.lrc_q4_apply(Q, s, None, X, None, Y, m, n, b, group, fmt)
    values = R.q4_values(Q, s, None, m, n, group)
    with_nan = X[:, :n].double() @ values.t()
    assert torch.equal(torch.isnan(Y.double()), torch.isnan(with_nan))
    assert torch.equal(torch.isinf(Y.double()), torch.isinf(with_nan))
    ok = torch.isfinite(with_nan)
    values[9] = 0
    x = X[:, :n].double().clone()
    x[b - 1] = 0
    want, bound = apply_bound(values, x, None, n, group, ot)
    off = torch.where(ok, (Y.double() - want).abs() - bound, torch.zeros_like(want))
    assert float(off.max()) <= 0


def test_apply_binary32_holds_binary32(lrc, cuda):
    """Vectors whose entries use all 24 bits, over 60 binary orders."""
    m, n, b, group = 64, 512, 4, 128
    Q, s, z = random_q4(cuda, m, n, group, True, "f32", 3)
    gen = torch.Generator(device=cuda).manual_seed(2)
    X = torch.randn((b, n), generator=gen, device=cuda) * torch.exp2(
        torch.randint(-30, 31, (b, n), generator=gen, device=cuda).float())
    Y = torch.empty((b, m), dtype=torch.float32, device=cuda)
    lrc.lrc_q4_apply(Q, s, z, X, None, Y, m, n, b, group, "f32")
    want, bound = apply_bound(R.q4_values(Q, s, z, m, n, group), X.double(), None, n, group, torch.float32)
    R.within(Y, want, bound)
    # one large entry, small ones beside it: what is left where they meet a zero code
    X = torch.full((1, n), 1.0 + 2.0 ** -23, device=cuda)
    X[0, 0] = 2.0 ** 100
    codes = R.q4_unpack(Q, n)
    codes[:, 0] = 8
    Y = torch.empty((1, m), dtype=torch.float32, device=cuda)
    lrc.lrc_q4_apply(R.q4_pack(codes), s, None, X, None, Y, m, n, 1, group, "f32")
    v = (codes.double() - 8) * R.spread(s, m, n, group)
    want, bound = apply_bound(v[:, 1:], X[:, 1:].double(), None, n, group, torch.float32)
    R.within(Y, want, bound)


def test_offsets_beyond_32_bits(lrc, cuda):
    """More than 2^32 bytes of codes: rows at the far end are right."""
    m, n, group, fmt = 140001, 65536, 128, "bf16"
    gen = torch.Generator(device=cuda).manual_seed(1)
    Q = torch.randint(0, 256, (m, n // 2), generator=gen, device=cuda, dtype=torch.uint8)
    s = torch.rand((n // group, R.ld16(m)), generator=gen, device=cuda).to(torch.bfloat16)
    X = torch.randn((2, n), generator=gen, device=cuda).to(torch.bfloat16)
    Y = torch.empty((2, m), dtype=torch.bfloat16, device=cuda)
    lrc.lrc_q4_apply(Q, s, None, X, None, Y, m, n, 2, group, fmt)
    rows = torch.tensor([0, 1, m // 2, m - 17, m - 1], device=cuda)
    v = R.q4_values(Q[rows], s[:, rows], None, len(rows), n, group)
    want, bound = apply_bound(v, X.double(), None, n, group, torch.bfloat16)
    R.within(Y[:, rows], want, bound)
    wide = torch.empty((m, n), dtype=torch.bfloat16, device=cuda)
    lrc.lrc_q4_widen(Q, s, None, group, fmt, m, n, wide, "bf16", n)
    assert torch.equal(wide[rows], v.float().to(torch.bfloat16))
    q = lrc.q4_matrix(wide, fmt, group)
    assert torch.equal(R.q4_unpack(q.Q[rows], n).cpu(),
                       torch.from_numpy(rounded_by_definition(wide[rows], group, False, torch.bfloat16)[0]))


def test_on_another_stream(lrc, cuda):
    m, n, b, group = 300, 700, 3, 64
    Q, s, z = random_q4(cuda, m, n, group, True, "f16", 8)
    X = torch.zeros((b, R.ld16(n)), dtype=torch.float16, device=cuda)
    X[:, :n] = torch.randn((b, n), device=cuda)
    ref = torch.empty((b, m), device=cuda)
    lrc.lrc_q4_apply(Q, s, z, X, None, ref, m, n, b, group, "f16")
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for i in range(8):
        Y = torch.full((b, m), float("nan"), device=cuda)
        streams[i % 2].wait_stream(torch.cuda.current_stream())
        lrc.lrc_q4_apply(Q, s, z, X, None, Y, m, n, b, group, "f16", stream=streams[i % 2])
        outs.append(Y)
    torch.cuda.synchronize()
    assert all(torch.equal(Y, ref) for Y in outs)


def test_in_a_graph(lrc, cuda):
    """Captured on its own stream and replayed on new vectors."""
    m, n, b, group = 200, 900, 2, 128
    Q, s, z = random_q4(cuda, m, n, group, False, "f32", 4)
    X = torch.randn((b, R.ld16(n)), device=cuda)
    Y, ref = torch.empty((b, m), device=cuda), torch.empty((b, m), device=cuda)
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        lrc.lrc_q4_apply(Q, s, z, X, None, Y, m, n, b, group, "f32")
    st.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        lrc.lrc_q4_apply(Q, s, z, X, None, Y, m, n, b, group, "f32")
    X.copy_(torch.randn((b, R.ld16(n)), device=cuda))
    graph.replay()
    lrc.lrc_q4_apply(Q, s, z, X, None, ref, m, n, b, group, "f32")
    torch.cuda.synchronize()
    assert torch.equal(Y, ref)


def test_no_vectors(lrc, cuda):
    Q, s, _ = random_q4(cuda, 4, 64, 32, False, "f32", 1)
    before = lrc.lrc_launch_count()
    lrc.lrc_q4_apply(Q, s, None, None, None, None, 4, 64, 0, 32, "f32")
    assert lrc.lrc_launch_count() == before
