"""What the operators around a compressed layer refuse, on the host: the C ABI
before any launch, the binding before the library.  And the codes' layout."""
import pytest
import torch

import layer_ref as R
import paper_2607_12969_gb300 as lrc
from test_abi import L                     # noqa: F401  (the fixture)
from test_binding_checks import AsCuda

F64, F32, F16, O16, TC, BF16 = range(6)
P = 4096                                   # an address that nothing reads


def test_row_bytes(L):                     # noqa: F811
    assert [lrc.lrc_q4_row_bytes(n) for n in (-1, 0, 1, 128, 129, 8192)] == [-1, 0, 64, 64, 128, 4096]


def test_layout_helpers_agree():
    g = torch.Generator().manual_seed(1)
    for n in (1, 7, 128, 300):
        c = torch.randint(0, 16, (5, n), generator=g)
        Q = R.q4_pack(c)
        assert Q.shape[1] == -(-n // 128) * 64 and torch.equal(R.q4_unpack(Q, n), c)
    # column 32 j + 8 t + e in word 4 t + j, bits from 4 NIBBLE[e] on
    c = torch.full((1, 128), 0, dtype=torch.int64)
    c[0, 32 * 2 + 8 * 3 + 5] = 9
    word = R.q4_pack(c).view(torch.int32)[0]
    assert int(word[4 * 3 + 2]) & 0xffffffff == 9 << (4 * 6) and int((word != 0).sum()) == 1


def test_q4_refusals(L):                   # noqa: F811
    ok = dict(Q=P, s=P, z=None, m=4, n=40, group=32, fmt=F16)

    def status(call, **kw):
        a = {**ok, **kw}
        if call == "round":
            return L.lrc_q4_round(a.get("W", P), a.get("wfmt", F32), a["m"], a["n"], a.get("ld", 40), a["Q"], a["s"],
                                  a["z"], a["group"], a["fmt"], None)
        if call == "widen":
            return L.lrc_q4_widen(a["Q"], a["s"], a["z"], a["group"], a["fmt"], a["m"], a["n"], a.get("dst", P),
                                  a.get("dfmt", F32), a.get("ld", 40), None)
        return L.lrc_q4_apply(a["Q"], a["s"], a["z"], a.get("X", P), a.get("A"), a.get("Y", P), a["m"], a["n"],
                              a.get("b", 1), a["group"], a["fmt"], None)

    for call in ("round", "widen", "apply"):
        assert status(call, Q=None) == -1 and status(call, s=None) == -1
        assert status(call, m=0) == -1 and status(call, n=-3) == -1 and status(call, group=0) == -1
        assert status(call, fmt=6) == -1 and status(call, fmt=-1) == -1
        assert status(call, fmt=F64) == -3 and status(call, group=48) == -3 and status(call, group=256) == -3
        assert status(call, Q=P + 8) == -2 and status(call, s=P + 2) == -2 and status(call, z=P + 1) == -2
        assert status(call, m=2 ** 62) == -1 and status(call, n=2 ** 62, ld=2 ** 62) == -1
        assert status(call, m=2 ** 63 - 1) == -1 and status(call, n=2 ** 63 - 1, ld=2 ** 63 - 1) == -1
    assert status("round", ld=39) == -1 and status("round", W=None) == -1 and status("round", W=P + 2) == -2
    assert status("round", wfmt=9) == -1 and status("round", W=P + 4, wfmt=F64) == -2
    assert status("widen", ld=39) == -1 and status("widen", dst=None) == -1 and status("widen", dst=P + 1) == -2
    assert status("widen", dfmt=7) == -1
    assert status("apply", b=-1) == -1 and status("apply", X=None) == -1 and status("apply", Y=None) == -1
    assert status("apply", X=P + 8) == -2 and status("apply", A=P + 4) == -2 and status("apply", Y=P + 2) == -2
    assert status("apply", b=0, X=None, Y=None) == 0
    assert status("apply", b=2 ** 62) == -1


def test_norm_refusals(L):                 # noqa: F811
    def norm(X=P, g=P, b=P, Y=P, mean=P, rstd=P, rows=2, cols=8, ldx=8, ldy=8, eps=1e-5, fmt=F32, pfmt=F32):
        return L.lrc_layer_norm(X, g, b, Y, mean, rstd, rows, cols, ldx, ldy, eps, fmt, pfmt, None)

    def grad(dY=P, X=P, g=P, mean=P, rstd=P, dX=P, dg=P, db=P, rows=2, cols=8, lddy=8, ldx=8, lddx=8, fmt=F32, pfmt=F32):
        return L.lrc_layer_norm_grad(dY, X, g, mean, rstd, dX, dg, db, rows, cols, lddy, ldx, lddx, fmt, pfmt, None)

    for f in (norm, grad):
        assert f(rows=-1) == -1 and f(cols=0) == -1 and f(rows=2 ** 31) == -1 and f(ldx=7) == -1
        assert f(fmt=6) == -1 and f(pfmt=-1) == -1 and f(fmt=F64) == -3 and f(pfmt=F64) == -3
        assert f(fmt=BF16, pfmt=F16) == -1 and f(fmt=F16, pfmt=BF16) == -1 and f(fmt=F32, pfmt=F16) == -1
        assert f(X=None) == -1 and f(X=P + 2) == -2 and f(g=P + 2) == -2 and f(rstd=P + 1) == -2 and f(mean=P + 3) == -2
        assert f(rows=2 ** 30, ldx=2 ** 40) == -1
    assert norm(Y=None) == -1 and norm(Y=P + 2, fmt=F16) == -2 and norm(ldy=7) == -1 and norm(b=P + 1) == -2
    assert norm(eps=-1.0) == -1 and norm(eps=float("nan")) == -1 and norm(eps=float("inf")) == -1 and norm(eps=1e39) == -1
    assert norm(rows=0, X=None, Y=None) == 0
    assert grad(dY=None) == -1 and grad(mean=None) == -1 and grad(rstd=None) == -1 and grad(lddy=7) == -1
    assert grad(lddx=7) == -1 and grad(dX=P + 2) == -2 and grad(dg=P + 2) == -2 and grad(db=P + 1) == -2
    assert grad(rows=0, dg=None, db=None) == 0


def test_distill_refusals(L):              # noqa: F811
    nan, inf = float("nan"), float("inf")

    def loss(Z=P, T=P, idx=P, w=None, loss=P, lse=P, dZ=P, rows=2, V=9, K=3, ldz=9, ldt=3, lddz=9, tau=1.0, fmt=F32,
             tfmt=F32):
        return L.lrc_distill(Z, T, idx, w, loss, lse, dZ, rows, V, K, ldz, ldt, lddz, tau, fmt, tfmt, None)

    def grad(Z=P, T=P, idx=P, w=None, lse=P, g=None, dZ=P, rows=2, V=9, K=3, ldz=9, ldt=3, lddz=9, tau=1.0, fmt=F32,
             tfmt=F32):
        return L.lrc_distill_grad(Z, T, idx, w, lse, g, dZ, rows, V, K, ldz, ldt, lddz, tau, fmt, tfmt, None)

    for f in (loss, grad):
        assert f(rows=-1) == -1 and f(V=0) == -1 and f(K=0) == -1 and f(rows=2 ** 31) == -1
        assert f(ldz=8) == -1 and f(ldt=2) == -1 and f(lddz=8) == -1
        assert f(tau=0.0) == -1 and f(tau=-1.0) == -1 and f(tau=nan) == -1 and f(tau=inf) == -1 and f(tau=1e-45) == -1
        assert f(fmt=6) == -1 and f(tfmt=-1) == -1 and f(fmt=F64) == -3 and f(tfmt=F64) == -3
        assert f(K=1025, ldt=1025) == -3
        assert f(Z=None) == -1 and f(T=None) == -1 and f(idx=None) == -1
        assert f(Z=P + 2) == -2 and f(T=P + 1) == -2 and f(idx=P + 4) == -2 and f(w=P + 2) == -2 and f(dZ=P + 1) == -2
        assert f(lse=P + 2) == -2 and f(rows=2 ** 30, ldz=2 ** 40) == -1
        assert f(rows=0, Z=None, T=None, idx=None) == 0
    assert loss(loss=P + 1) == -2 and loss(loss=None, lse=None, dZ=None) == 0
    assert grad(lse=None) == -1 and grad(dZ=None) == -1 and grad(g=P + 2) == -2


class Stand(AsCuda):
    """With an address: a call whose other arguments are wrong takes it, and goes no further."""

    def data_ptr(self):
        return P


@pytest.fixture
def current_device_0(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)


def test_binding_refusals(current_device_0):
    h = lambda shape, dt=torch.float32: Stand(torch.zeros(shape, dtype=dt))      # noqa: E731
    Q, s, z = h((4, 64), torch.uint8), h((2, 16)), h((2, 16), torch.uint8)
    with pytest.raises(ValueError, match="CUDA tensor"):
        lrc.lrc_q4_apply(torch.zeros((4, 64), dtype=torch.uint8), s, z, h((1, 64)), None, h((1, 4)), 4, 60, 1, 32, "f32")
    with pytest.raises(ValueError, match="Q: storage holds"):
        lrc.lrc_q4_apply(h((3, 64), torch.uint8), s, z, h((1, 64)), None, h((1, 4)), 4, 60, 1, 32, "f32")
    with pytest.raises(ValueError, match="scales: storage holds"):
        lrc.lrc_q4_apply(Q, h((1, 16)), z, h((1, 64)), None, h((1, 4)), 4, 60, 1, 32, "f32")
    with pytest.raises(ValueError, match="zeros: element type"):
        lrc.lrc_q4_apply(Q, s, h((2, 16)), h((1, 64)), None, h((1, 4)), 4, 60, 1, 32, "f32")
    with pytest.raises(ValueError, match="X: storage holds"):
        lrc.lrc_q4_apply(Q, s, z, h((1, 59)), None, h((1, 4)), 4, 60, 1, 32, "f32")
    with pytest.raises(ValueError, match="A: storage holds"):
        lrc.lrc_q4_apply(Q, s, z, h((1, 64)), h((1, 3)), h((1, 4)), 4, 60, 1, 32, "f32")
    with pytest.raises(ValueError, match="W: storage holds"):
        lrc.lrc_q4_round(h((4, 59)), "f32", 4, 60, 60, Q, s, z, 32, "f32")
    with pytest.raises(ValueError, match="dst: element type"):
        lrc.lrc_q4_widen(Q, s, z, 32, "f32", 4, 60, h((4, 60)), "f16", 60)
    with pytest.raises(ValueError, match="mean: storage holds"):
        lrc.lrc_layer_norm(h((4, 8)), None, None, h((4, 8)), h((3,)), None, 4, 8, 8, 8, 1e-5, "f32", "f32")
    with pytest.raises(ValueError, match="Y: storage holds"):
        lrc.lrc_layer_norm(h((4, 8)), None, None, h((4, 8)), None, None, 4, 8, 8, 9, 1e-5, "f32", "f32")
    with pytest.raises(ValueError, match="gamma: element type"):
        lrc.lrc_layer_norm(h((4, 8)), h((8,)), None, h((4, 8)), None, None, 4, 8, 8, 8, 1e-5, "f32", "bf16")
    with pytest.raises(ValueError, match="dgamma: storage holds"):
        lrc.lrc_layer_norm_grad(h((4, 8)), h((4, 8)), None, h((4,)), h((4,)), None, h((7,)), None, 4, 8, 8, 8, 8, "f32",
                                "f32")
    with pytest.raises(ValueError, match="rstd: a tensor is required"):
        lrc.lrc_layer_norm_grad(h((4, 8)), h((4, 8)), None, h((4,)), None, None, h((8,)), None, 4, 8, 8, 8, 8, "f32",
                                "f32")
    i = h((2, 3), torch.int64)
    with pytest.raises(ValueError, match="idx: element type"):
        lrc.lrc_distill(h((2, 9)), h((2, 3)), h((2, 3)), None, None, h((2,)), None, 2, 9, 3, 9, 3, 9, 1.0, "f32", "f32")
    with pytest.raises(ValueError, match="dZ: storage holds"):
        lrc.lrc_distill(h((2, 9)), h((2, 3)), i, None, None, h((2,)), h((2, 8)), 2, 9, 3, 9, 3, 9, 1.0, "f32", "f32")
    with pytest.raises(ValueError, match="loss: storage holds"):
        lrc.lrc_distill(h((2, 9)), h((2, 3)), i, None, h((1,)), None, None, 2, 9, 3, 9, 3, 9, 1.0, "f32", "f32")
    with pytest.raises(ValueError, match="dZ: a tensor is required"):
        lrc.lrc_distill_grad(h((2, 9)), h((2, 3)), i, None, h((2,)), None, None, 2, 9, 3, 9, 3, 9, 1.0, "f32", "f32")
