"""What the operators around a compressed layer are judged on.

A program that keeps a layer's weights in few bits -- 4-bit codes with group
scales, beside the low-rank factors that compensate them -- needs, next to the
low-rank apply,

* the codes themselves (rounding a matrix to 4 bits, and its values back for
  the perturbation eta) and the product of such a matrix with one or a few
  vectors, which is what a server does for every token;
* layer norm and its gradient: what is trained again, with the matrices
  frozen, after they were rounded;
* the distillation loss against the top logits that the original model gave,
  with its gradient: what that training minimises.

Sizes are those of the benchmark's workloads and of the tests (matrices with
sides of 512, 8192 and 16384, odd sides near them, batches of 1 to 64 vectors)
or plain powers of two and odd numbers.
"""
import math

import torch

own = False

DEV = "cuda:0"

_STORE = {"f32": torch.float32, "f16": torch.float16, "f16_o16": torch.float16, "bf16": torch.bfloat16}
_OUT = {"f32": torch.float32, "f16": torch.float32, "f16_o16": torch.float16, "bf16": torch.bfloat16}


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------

def listed():
    return [
        # storing the matrix of the smallest configuration: latency
        dict(name="q4_store_small", kind="store", m=512, n=512, src="f32", fmt="f16", group=32, zeros=False),
        # storing the large configuration's matrix and widening it for eta
        dict(name="q4_store_large", kind="store", m=16384, n=8192, src="bf16", fmt="bf16", group=128, zeros=True),
        # one token through a small layer: latency
        dict(name="q4_token_small", kind="apply", m=512, n=512, b=1, fmt="f16", group=32, zeros=False, add=False),
        # one token through a large layer: the weights' bytes
        dict(name="q4_token_large", kind="apply", m=16384, n=16384, b=1, fmt="bf16", group=128, zeros=False,
             add=False),
        # a few tokens in binary32, a matrix with odd sides, asymmetric codes,
        # on top of the low-rank part's result
        dict(name="q4_odd_f32", kind="apply", m=12287, n=16381, b=7, fmt="f32", group=64, zeros=True, add=True),
        # a server's batch of 64 on top of the low-rank part
        dict(name="q4_batch_f16o16", kind="apply", m=16384, n=8192, b=64, fmt="f16_o16", group=128, zeros=False,
             add=True),
        # the norm before a layer while it serves a batch
        dict(name="norm_serve_f16", kind="norm", rows=64, cols=8192, pad=0, fmt="f16", pfmt="f16"),
        # its gradient in a training step, weights kept in binary32
        dict(name="norm_grad_bf16", kind="norm_grad", rows=8192, cols=8192, pad=0, fmt="bf16", pfmt="f32"),
        # an odd width, rows cut out of a wider array
        dict(name="norm_grad_odd_f32", kind="norm_grad", rows=4099, cols=1138, pad=7, fmt="f32", pfmt="f32"),
        # scoring a few answers against the teacher: forward only
        dict(name="distill_score_f32", kind="distill", rows=16, V=32768, K=32, pad=0, fmt="f32", tfmt="f32", tau=1.0,
             grad=False),
        # a training step's loss and gradient at once
        dict(name="distill_step_bf16", kind="distill", rows=4096, V=65536, K=64, pad=0, fmt="bf16", tfmt="f16",
             tau=2.0, grad=True),
        # the gradient apart (an upstream gradient per row), an odd vocabulary
        # whose rows start at odd addresses
        dict(name="distill_grad_odd_f16", kind="distill_grad", rows=1021, V=50001, K=17, pad=0, fmt="f16", tfmt="f32",
             tau=1.5),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges above."""
    kind = rng.choice(["store", "apply", "apply", "apply", "norm", "norm_grad", "distill", "distill_grad"])
    fmt = rng.choice(["f32", "f16", "f16_o16", "bf16"])
    if kind == "store":
        m, n = _log_int(rng, 512, 16384), _log_int(rng, 512, 8192)
        return dict(kind=kind, m=m, n=n, src=rng.choice(["f32", "f16", "bf16"]), fmt=rng.choice(["f32", "f16", "bf16"]),
                    group=rng.choice([32, 64, 128]), zeros=rng.random() < 0.5)
    if kind == "apply":
        m, n = _log_int(rng, 512, 16384), _log_int(rng, 512, 16384)
        b = _log_int(rng, 1, 64)
        b = max(1, min(b, 16384 * 8192 * 64 // (m * n)))
        return dict(kind=kind, m=m, n=n, b=b, fmt=fmt, group=rng.choice([32, 64, 128]), zeros=rng.random() < 0.5,
                    add=rng.random() < 0.5)
    if kind in ("norm", "norm_grad"):
        rows, cols = _log_int(rng, 1, 8192), _log_int(rng, 256, 16384)
        rows = max(1, min(rows, 8192 * 8192 * (1 if fmt in ("f16_o16", "bf16") else 2) // (2 * cols)))
        return dict(kind=kind, rows=rows, cols=cols, pad=rng.choice([0, 0, 7, 16]), fmt=fmt,
                    pfmt="f32" if fmt == "f32" or rng.random() < 0.5 else fmt)
    V = _log_int(rng, 4096, 262144)
    if rng.random() < 0.5:
        V = max(64, V // 64 * 64)
    fmt = rng.choice(["f32", "f16", "bf16"])
    rows = max(1, min(_log_int(rng, 1, 8192), 4096 * 65536 // V // (2 if fmt == "f32" else 1)))
    c = dict(kind=kind, rows=rows, V=V, K=_log_int(rng, 1, 256), pad=rng.choice([0, 0, 5, 16]), fmt=fmt,
             tfmt=rng.choice(["f32", "f16"]), tau=rng.choice([1.0, 1.5, 2.0, 4.0]))
    if kind == "distill":
        c["grad"] = rng.random() < 0.6
    return c


# ---------------------------------------------------------------------------
# what a program has in hand
# ---------------------------------------------------------------------------

def _ld(cols):
    return (cols + 15) // 16 * 16


# Codes lie in rows of 64-byte blocks, 128 columns each.  Within a block, column
# 32 j + 8 t + e (j, t < 4, e < 8) is in the 32-bit word 4 t + j, at the four
# bits from 4 _NIBBLE[e] on.
_NIBBLE = [0, 4, 1, 5, 2, 6, 3, 7]
_COLUMN = [0, 2, 4, 6, 1, 3, 5, 7]


def _lay_out(codes, m, n):
    """Codes 0 ... 15 (m x n128, one a byte) in that layout."""
    c = codes.view(m, -1, 4, 4, 8)[..., _COLUMN].transpose(2, 3)
    return (c[..., 0::2] | (c[..., 1::2] << 4)).reshape(m, -1).contiguous()


def _codes(Q, m, n):
    """The codes of a laid-out matrix, m x n."""
    q = Q.view(m, -1, 4, 4, 4)
    c = torch.stack([q & 15, q >> 4], -1).view(m, -1, 4, 4, 8)[..., _NIBBLE]
    return c.transpose(2, 3).reshape(m, -1)[:, :n]


def _logits(shape, gen):
    """Logits as a model gives them: a few large ones above a broad floor."""
    z = torch.randn(shape, generator=gen, device=DEV)
    return z.mul_(1.5).add_(0.02 * z ** 3)


def _normal(shape, gen, dtype=torch.float32):
    return torch.randn(shape, generator=gen, device=DEV).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    st = dict(case)
    kind, fmt = case["kind"], case["fmt"]
    dt, ot = _STORE[fmt], _OUT[fmt]
    if kind in ("store", "apply"):
        m, n, group = case["m"], case["n"], case["group"]
        groups, ldm = -(-n // group), _ld(m)
        st["groups"] = groups
        zeros = case["zeros"]
    if kind == "store":
        W = torch.randn((m, n), generator=gen, device=DEV)
        W *= 0.02 * (0.5 + torch.rand((m, 1), generator=gen, device=DEV))
        st["W"] = W.to(_STORE[case["src"]])
        st["Q"] = torch.empty((m, -(-n // 128) * 64), dtype=torch.uint8, device=DEV)
        st["scales"] = torch.zeros((groups, ldm), dtype=dt, device=DEV)
        st["zeros_out"] = torch.zeros((groups, ldm), dtype=torch.uint8, device=DEV) if zeros else None
        st["values"] = torch.empty((m, n), dtype=torch.float32, device=DEV)
    elif kind == "apply":
        b, nb = case["b"], -(-n // 128) * 128
        Q = torch.empty((m, nb // 2), dtype=torch.uint8, device=DEV)
        for r in range(0, m, 4096):      # in blocks of rows, to spare memory
            c = torch.randn((min(4096, m - r), nb), generator=gen, device=DEV)
            c[:, n:] = 0
            c = c.mul_(2.4).round_().add_(8).clamp_(0, 15).to(torch.uint8)
            Q[r:r + 4096] = _lay_out(c, c.shape[0], n)
        st["Q"] = Q
        s = torch.rand((groups, ldm), generator=gen, device=DEV).add_(0.5).mul_(n ** -0.5 / 2.4)
        st["scales"] = s.to(dt)
        st["zeros_in"] = torch.randint(5, 11, (groups, ldm), generator=gen, device=DEV).to(torch.uint8) if zeros else None
        X = torch.zeros((b, _ld(n)), dtype=dt, device=DEV)
        X[:, :n] = _normal((b, n), gen)
        st["X"] = X
        st["A"] = _normal((b, m), gen, ot) if case["add"] else None
        st["Y"] = torch.empty((b, m), dtype=ot, device=DEV)
    elif kind in ("norm", "norm_grad"):
        rows, cols, ld = case["rows"], case["cols"], case["cols"] + case["pad"]
        pdt = _STORE[case["pfmt"]]
        X = _normal((rows, ld), gen) * (0.5 + 2 * torch.rand((1, ld), generator=gen, device=DEV))
        X += 0.5 + 0.2 * _normal((rows, 1), gen)
        st["X"] = X.to(dt)
        st["ld"] = ld
        st["gamma"] = (1 + 0.2 * _normal((cols,), gen)).to(pdt)
        st["beta"] = (0.1 * _normal((cols,), gen)).to(pdt)
        if kind == "norm":
            st["Y"] = torch.empty((rows, cols), dtype=ot, device=DEV)
            st["mean"] = torch.empty(rows, dtype=torch.float32, device=DEV)
            st["rstd"] = torch.empty(rows, dtype=torch.float32, device=DEV)
        else:
            x = st["X"][:, :cols].double()
            mean = x.mean(1)
            st["mean"] = mean.float()
            st["rstd"] = (x.var(1, unbiased=False) + 1e-5).rsqrt().float()
            st["dY"] = (_normal((rows, ld), gen) * 0.3 + 0.1).to(ot)
            st["dX"] = torch.empty((rows, cols), dtype=dt, device=DEV)
            st["dgamma"] = torch.empty(cols, dtype=torch.float32, device=DEV)
            st["dbeta"] = torch.empty(cols, dtype=torch.float32, device=DEV)
    else:
        rows, V, K, ld = case["rows"], case["V"], case["K"], case["V"] + case["pad"]
        tdt = _STORE[case["tfmt"]]
        Z = torch.empty((rows, ld), dtype=dt, device=DEV)
        idx = torch.empty((rows, K), dtype=torch.int64, device=DEV)
        T = torch.empty((rows, K), dtype=tdt, device=DEV)
        st["lse"] = torch.empty(rows, dtype=torch.float32, device=DEV)
        shut = torch.rand(ld, generator=gen, device=DEV) < 1e-3      # entries that may not be answered with
        for r in range(0, rows, 512):
            z = _logits((min(512, rows - r), ld), gen).masked_fill_(shut, -math.inf)
            teacher = z[:, :V] + 0.5 * _normal((z.shape[0], V), gen)
            top = torch.topk(teacher, K, dim=1)
            T[r:r + 512], idx[r:r + 512] = top.values, top.indices
            Z[r:r + 512] = z
            if kind == "distill_grad":
                st["lse"][r:r + 512] = torch.logsumexp(Z[r:r + 512, :V].double() / case["tau"], 1).float()
        # short lists end in -1; some rows have none, some have no weight (padding)
        short = torch.rand((rows, 1), generator=gen, device=DEV)
        keep = torch.where(short < 0.2, 1 + (K * torch.rand((rows, 1), generator=gen, device=DEV)).long(), K)
        keep = torch.where(short < 0.02, 0, keep)
        idx[torch.arange(K, device=DEV)[None, :] >= keep] = -1
        w = torch.rand(rows, generator=gen, device=DEV) + 0.5
        w[torch.rand(rows, generator=gen, device=DEV) < 0.05] = 0
        if dt == torch.float16:
            w *= 1024      # the loss scale that gradients in binary16 need
        st.update(Z=Z, T=T, idx=idx, w=w / rows, ld=ld)
        st["loss"] = torch.empty(rows, dtype=torch.float32, device=DEV)
        st["dZ"] = torch.empty((rows, V), dtype=dt, device=DEV) if kind == "distill_grad" or case["grad"] else None
        st["g"] = torch.rand(rows, generator=gen, device=DEV) + 0.5 if kind == "distill_grad" else None
    return st


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(st):
    return _run_own(st) if own else _run_plain(st)


def _run_own(st):
    import paper_2607_12969_gb300 as lrc
    kind, fmt = st["kind"], st["fmt"]
    if kind == "store":
        m, n = st["m"], st["n"]
        lrc.lrc_q4_round(st["W"], st["src"], m, n, n, st["Q"], st["scales"], st["zeros_out"], st["group"], fmt)
        lrc.lrc_q4_widen(st["Q"], st["scales"], st["zeros_out"], st["group"], fmt, m, n, st["values"], "f32", n)
        return [st["values"], st["scales"][:, :m]] + ([st["zeros_out"][:, :m]] if st["zeros"] else [])
    if kind == "apply":
        lrc.lrc_q4_apply(st["Q"], st["scales"], st["zeros_in"], st["X"], st["A"], st["Y"], st["m"], st["n"], st["b"],
                         st["group"], fmt)
        return [st["Y"]]
    if kind == "norm":
        lrc.lrc_layer_norm(st["X"], st["gamma"], st["beta"], st["Y"], st["mean"], st["rstd"], st["rows"], st["cols"],
                           st["ld"], st["cols"], 1e-5, fmt, st["pfmt"])
        return [st["Y"], st["mean"], st["rstd"]]
    if kind == "norm_grad":
        lrc.lrc_layer_norm_grad(st["dY"], st["X"], st["gamma"], st["mean"], st["rstd"], st["dX"], st["dgamma"],
                                st["dbeta"], st["rows"], st["cols"], st["ld"], st["ld"], st["cols"], fmt, st["pfmt"])
        return [st["dX"], st["dgamma"], st["dbeta"]]
    if kind == "distill":
        lrc.lrc_distill(st["Z"], st["T"], st["idx"], st["w"], st["loss"], st["lse"], st["dZ"], st["rows"], st["V"],
                        st["K"], st["ld"], st["K"], st["V"], st["tau"], fmt, st["tfmt"])
        return [st["loss"], st["lse"]] + ([st["dZ"]] if st["grad"] else [])
    lrc.lrc_distill_grad(st["Z"], st["T"], st["idx"], st["w"], st["lse"], st["g"], st["dZ"], st["rows"], st["V"],
                         st["K"], st["ld"], st["K"], st["V"], st["tau"], fmt, st["tfmt"])
    return [st["dZ"]]


def _per_column(a, m, n, group):
    """Group values (groups x m) spread over the columns of their groups: m x n."""
    return a[:, :m].float().t().repeat_interleave(group, 1)[:, :n]


def _round_plain(W, m, n, group, zeros, dt):
    """Codes, scales (as stored) and zero codes of a matrix, binary32 arithmetic."""
    groups = -(-n // group)
    w = torch.zeros((m, groups * group), device=DEV)
    w[:, :n] = W
    w = w.view(m, groups, group)
    if zeros:
        lo, hi = w.amin(2).clamp(max=0), w.amax(2).clamp(min=0)
        s = (hi - lo) * (1 / 15)
    else:
        s = w.abs().amax(2) * (1 / 7)
    s = s.clamp(max=torch.finfo(dt).max).to(dt)
    none = s.float() < 2.0 ** -126
    s = torch.where(none, torch.zeros_like(s), s)
    inv = torch.where(none, 0.0, torch.reciprocal(s.float()))
    z = torch.round(-lo * inv).clamp(0, 15) if zeros else torch.full_like(inv, 8)
    q = (torch.round(w * inv[..., None]) + z[..., None]).clamp(0, 15)
    return q.view(m, -1)[:, :n], s.t(), z.t()


def _run_plain(st):
    kind, fmt = st["kind"], st["fmt"]
    dt, ot = _STORE[fmt], _OUT[fmt]
    if kind == "store":
        m, n, group = st["m"], st["n"], st["group"]
        q, s, z = _round_plain(st["W"].float(), m, n, group, st["zeros"], dt)
        values = _per_column(s, m, n, group) * (q - _per_column(z, m, n, group))
        return [values, s] + ([z.to(torch.uint8)] if st["zeros"] else [])
    if kind == "apply":
        m, n, group = st["m"], st["n"], st["group"]
        z = 8 if st["zeros_in"] is None else _per_column(st["zeros_in"], m, n, group)
        W = (_codes(st["Q"], m, n).float() - z) * _per_column(st["scales"], m, n, group)
        Y = st["X"][:, :n].float() @ W.t()
        return [(Y if st["A"] is None else Y + st["A"].float()).to(ot)]
    if kind == "norm":
        x = st["X"][:, :st["cols"]].float()
        mean = x.mean(1)
        x = x - mean[:, None]
        rstd = torch.rsqrt((x * x).mean(1) + 1e-5)
        return [(x * rstd[:, None] * st["gamma"].float() + st["beta"].float()).to(ot), mean, rstd]
    if kind == "norm_grad":
        cols = st["cols"]
        xh = (st["X"][:, :cols].float() - st["mean"][:, None]) * st["rstd"][:, None]
        dy = st["dY"][:, :cols].float()
        d = dy * st["gamma"].float()
        dx = (d - d.mean(1, keepdim=True) - xh * (d * xh).mean(1, keepdim=True)) * st["rstd"][:, None]
        return [dx.to(dt), (dy * xh).sum(0), dy.sum(0)]
    V, tau, w, idx = st["V"], st["tau"], st["w"], st["idx"]
    z = st["Z"][:, :V].float() / tau
    there = (idx >= 0) & (idx < V)
    t = torch.where(there, st["T"].float() / tau, float("-inf"))
    top = t.amax(1, keepdim=True)
    on = (top[:, 0] > float("-inf")) & (w != 0)
    p = torch.where(on[:, None], torch.exp(t - top), 0.0)
    total = torch.where(on, p.sum(1), 1.0)
    p = p / total[:, None]
    at = idx.clamp(0, V - 1)
    out = []
    if kind == "distill":
        zmax = z.amax(1, keepdim=True)
        lse = torch.log(torch.exp(z - zmax).sum(1)) + zmax[:, 0]
        lp = t - top - torch.log(total)[:, None]
        lq = torch.gather(z, 1, at) - lse[:, None]
        kl = torch.where(p > 0, p * (lp - lq), 0.0).sum(1)
        out = [torch.where(on, tau * tau * w * kl, 0.0), lse]
        if not st["grad"]:
            return out
        g = tau * w
    else:
        lse = st["lse"]
        g = tau * w * st["g"]
    dz = torch.exp(z - lse[:, None])
    dz.scatter_add_(1, at, -p)
    return out + [torch.where(on[:, None], dz * g[:, None], 0.0).to(dt)]


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

_BYTES = {"f32": 4, "f16": 2, "f16_o16": 2, "bf16": 2}
_OUT_BYTES = {"f32": 4, "f16": 4, "f16_o16": 2, "bf16": 2}


def work(case):
    kind, e, o = case["kind"], _BYTES[case["fmt"]], _OUT_BYTES[case["fmt"]]
    if kind in ("store", "apply"):
        m, n = case["m"], case["n"]
        weights = m * n // 2 + m * -(-n // case["group"]) * (e + (1 if case["zeros"] else 0))
    if kind == "store":
        # the matrix read, the codes written and read again, their values written
        return {"bytes": m * n * (_BYTES[case["src"]] + 4) + 2 * weights, "flops": 6 * m * n}
    if kind == "apply":
        b = case["b"]
        return {"bytes": weights + b * n * e + b * m * o * (2 if case["add"] else 1), "flops": 2 * m * n * b}
    if kind in ("norm", "norm_grad"):
        rows, cols, p = case["rows"], case["cols"], _BYTES[case["pfmt"]]
        if kind == "norm":
            return {"bytes": rows * cols * (e + o) + rows * 8 + 2 * cols * p, "flops": 8 * rows * cols}
        return {"bytes": rows * cols * (2 * e + o) + rows * 8 + cols * (p + 8), "flops": 15 * rows * cols}
    rows, V, K = case["rows"], case["V"], case["K"]
    grad = kind == "distill_grad" or case["grad"]
    return {"bytes": rows * V * e * (2 if grad else 1) + rows * K * (8 + _BYTES[case["tfmt"]]) + 16 * rows,
            "flops": rows * V * (8 if grad else 5)}


# ---------------------------------------------------------------------------
# the same in 64 bits
# ---------------------------------------------------------------------------

def _exact_rounded(W, m, n, group, zeros, dt):
    """Values, scales and zero codes of a rounded matrix, group by group of columns."""
    values = torch.empty((m, n), dtype=torch.float64, device=DEV)
    scales, zero = [], []
    for c in range(0, n, group):
        w = W[:, c:c + group].double()
        if zeros:
            low = torch.minimum(w.min(1).values, torch.zeros((), dtype=torch.float64, device=DEV))
            high = torch.maximum(w.max(1).values, torch.zeros((), dtype=torch.float64, device=DEV))
            s = ((high - low) / 15).float().to(dt).double()
            z = torch.where(s > 0, torch.round(-low / s), 0.0).clamp(0, 15)
        else:
            s = (w.abs().max(1).values / 7).float().to(dt).double()
            z = torch.full_like(s, 8)
        k = torch.where(s[:, None] > 0, torch.round(w / s[:, None]), 0.0) + z[:, None]
        values[:, c:c + group] = (k.clamp(0, 15) - z[:, None]) * s[:, None]
        scales.append(s)
        zero.append(z)
    return values, torch.stack(scales), torch.stack(zero)


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "store":
        values, s, z = _exact_rounded(st["W"], st["m"], st["n"], st["group"], st["zeros"], _STORE[st["fmt"]])
        return [values, s] + ([None] if st["zeros"] else [])
    if kind == "apply":
        m, n, group = st["m"], st["n"], st["group"]
        words = st["Q"].view(torch.int32)
        x = st["X"].double()
        Y = torch.zeros((st["b"], m), dtype=torch.float64, device=DEV) if st["A"] is None else st["A"].double()
        step = 2048
        for r in range(0, m, step):
            rows = words[r:r + step]
            W = torch.zeros((rows.shape[0], rows.shape[1] * 8), dtype=torch.float64, device=DEV)
            part = W.view(rows.shape[0], -1, 4, 4, 8)
            for e in range(8):
                part[..., e] = ((rows >> (4 * _NIBBLE[e])) & 15).view(rows.shape[0], -1, 4, 4).transpose(2, 3)
            for g in range(st["groups"]):
                z = 8 if st["zeros_in"] is None else st["zeros_in"][g, r:r + step, None][:rows.shape[0]].double()
                cut = W[:, g * group:(g + 1) * group]
                cut.sub_(z).mul_(st["scales"][g, r:r + step, None][:rows.shape[0]].double())
            Y[:, r:r + step] += x[:, :n] @ W[:, :n].t()
        return [Y]
    if kind == "norm":
        x = st["X"][:, :st["cols"]].double()
        var, mean = torch.var_mean(x, 1, unbiased=False)
        rstd = 1 / torch.sqrt(var + 1e-5)
        return [(x - mean[:, None]) * (rstd[:, None] * st["gamma"].double()) + st["beta"].double(), mean, rstd]
    if kind == "norm_grad":
        n = st["cols"]
        r = st["rstd"].double()[:, None]
        xh = (st["X"][:, :n].double() - st["mean"].double()[:, None]) * r
        dy = st["dY"][:, :n].double()
        dg = torch.einsum("rc,rc->c", dy, xh)
        dy_g = dy * st["gamma"].double()
        a = torch.einsum("rc,rc->r", dy_g, xh)[:, None] / n
        return [r * (dy_g - dy_g.sum(1, keepdim=True) / n - a * xh), dg, dy.sum(0)]
    V, K, tau, rows = st["V"], st["K"], st["tau"], st["rows"]
    grad = kind == "distill_grad" or case["grad"]
    loss = torch.zeros(rows, dtype=torch.float64, device=DEV)
    lse = torch.empty(rows, dtype=torch.float64, device=DEV)
    dZ = torch.empty((rows, V), dtype=torch.float64, device=DEV) if grad else None
    for r in range(0, rows, 256):
        cut = slice(r, min(r + 256, rows))
        z = st["Z"][cut, :V].double() / tau
        lse[cut] = st["lse"][cut].double() if kind == "distill_grad" else torch.logsumexp(z, 1)
        logq = z - lse[cut, None]
        i = st["idx"][cut]
        t = (st["T"][cut].double() / tau).masked_fill((i < 0) | (i >= V), -math.inf)
        logp = torch.log_softmax(t, 1)
        p = logp.exp().nan_to_num(0.0)
        w = st["w"][cut].double() * (p.sum(1) > 0)
        P = torch.zeros_like(z)
        P.scatter_add_(1, i.clamp(0, V - 1), p)
        each = logp.nan_to_num(0.0, neginf=0.0) - logq.gather(1, i.clamp(0, V - 1))
        loss[cut] = tau ** 2 * w * torch.where(p > 0, p * each, 0.0).sum(1)
        if grad:
            up = tau * w * (st["g"][cut].double() if kind == "distill_grad" else 1.0)
            dZ[cut] = (logq.exp() - P) * up[:, None]
    if kind == "distill_grad":
        return [dZ]
    return [loss, lse] + ([dZ] if grad else [])
