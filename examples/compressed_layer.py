"""A compressed layer, served and repaired.

A small model -- a dense layer, layer norm, an output head -- is compressed: the
layer's matrix becomes 4-bit codes with group scales, and the truncated SVD of
what the codes leave over is stored in binary16 beside them (rank compensation);
the head is kept as low-rank factors.  Then

* served: one token through the codes and the compensating factors,
* repaired: with every matrix frozen, the norm's gamma and beta are trained on
  the distillation loss against the top logits of the uncompressed model.  The
  gradient passes the head as an apply of its factors exchanged.

Run:  python examples/compressed_layer.py
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2607_12969_gb300 as lrc  # noqa: E402


def factors(A, k, fmt):
    """Rank-k factors of A in format fmt: (U, S, Vt) as lrc_apply takes them, and
    those of A^T."""
    U, s, Vt = torch.linalg.svd(A.double(), full_matrices=False)
    U, s, Vt = U[:, :k].contiguous(), s[:k].contiguous(), Vt[:k].contiguous()
    S = lrc.round_matrix(s[None, :], fmt)
    return ((lrc.round_matrix(U, fmt), S, lrc.round_matrix(Vt, fmt)),
            (lrc.round_matrix(Vt.t().contiguous(), fmt), S, lrc.round_matrix(U.t().contiguous(), fmt)))


class Layer:
    """An m x n matrix as 4-bit codes plus rank-k factors of what they leave over."""

    def __init__(self, W, k, group=64, fmt="f16"):
        self.m, self.n = W.shape
        self.k, self.fmt = k, fmt
        self.q = lrc.q4_matrix(W, fmt, group, zeros=True)
        What = torch.empty((self.m, self.n), dtype=torch.float64, device=W.device)
        lrc.lrc_q4_widen(self.q.Q, self.q.scales, self.q.zeros, group, fmt, self.m, self.n, What, "f64", self.n)
        self.eta, norm = lrc.lrc_fro_diff(W.double().contiguous(), "f64", What, "f64", What.numel())
        self.eta /= norm
        self.low = factors(W.double() - What, k, fmt)[0]

    def __call__(self, X, compensate=True):
        """b x n vectors (packed pitch, the storage type) to b x m results."""
        b, q = X.shape[0], self.q
        Y = torch.empty((b, self.m), dtype=lrc.output_dtype(self.fmt), device=X.device)
        if compensate:
            lrc.lrc_apply(*self.low, X, Y, self.m, self.n, self.k, b, self.fmt)
        lrc.lrc_q4_apply(q.Q, q.scales, q.zeros, X, Y if compensate else None, Y, self.m, self.n, b, q.group, self.fmt)
        return Y


class Repair:
    """Training of gamma and beta between the frozen layer and the frozen head."""

    def __init__(self, layer, head, V, k, top, at, X, tau):
        (self.head, self.head_t), self.V, self.k, self.tau = head, V, k, tau
        self.m, self.rows = layer.m, X.shape[0]
        dev = X.device
        self.H = layer(X)                                         # frozen: one pass is enough
        self.gamma, self.beta = torch.ones(self.m, device=dev), torch.zeros(self.m, device=dev)
        self.top, self.at = top, at
        self.N = torch.zeros((self.rows, lrc.lrc_packed_ld(self.m)), device=dev)
        self.mean, self.rstd, self.loss, self.lse = (torch.empty(self.rows, device=dev) for _ in range(4))
        self.Z = torch.empty((self.rows, V), device=dev)
        self.dZ = torch.zeros((self.rows, lrc.lrc_packed_ld(V)), device=dev)
        self.dN = torch.empty((self.rows, self.m), device=dev)
        self.grads = torch.empty(self.m, device=dev), torch.empty(self.m, device=dev)
        self.w = torch.full((self.rows,), 1.0 / self.rows, device=dev)
        self.adam = [torch.zeros_like(t) for t in (self.gamma, self.gamma, self.beta, self.beta)]
        self.t = 0

    def step(self, lr):
        """One step of Adam; returns the loss before it."""
        rows, m, V, k, ldn, ldv = self.rows, self.m, self.V, self.k, self.N.shape[1], self.dZ.shape[1]
        lrc.lrc_layer_norm(self.H, self.gamma, self.beta, self.N, self.mean, self.rstd, rows, m, m, ldn, 1e-5, "f32", "f32")
        lrc.lrc_apply(*self.head, self.N, self.Z, V, m, k, rows, "f32")
        lrc.lrc_distill(self.Z, self.top, self.at, self.w, self.loss, self.lse, self.dZ, rows, V, self.top.shape[1], V,
                        self.top.shape[1], ldv, self.tau, "f32", "f32")
        lrc.lrc_apply(*self.head_t, self.dZ, self.dN, m, V, k, rows, "f32")
        lrc.lrc_layer_norm_grad(self.dN, self.H, self.gamma, self.mean, self.rstd, None, *self.grads, rows, m, m, m, m,
                                "f32", "f32")
        self.t += 1
        for p, g, a, b in zip((self.gamma, self.beta), self.grads, self.adam[::2], self.adam[1::2]):
            a.mul_(0.9).add_(g, alpha=0.1)
            b.mul_(0.99).addcmul_(g, g, value=0.01)
            p.sub_(lr * (a / (1 - 0.9 ** self.t)) / ((b / (1 - 0.99 ** self.t)).sqrt() + 1e-8))
        return float(self.loss.sum())


def main(m=512, n=512, V=2000, rows=256, k=32, head_rank=256, top=32, steps=40, seed=1):
    dev = torch.device("cuda:0")
    g = torch.Generator(device=dev).manual_seed(seed)
    W = torch.randn((m, n), generator=g, device=dev) / n ** 0.5
    W *= torch.exp(0.5 * torch.randn((m, 1), generator=g, device=dev))
    head = torch.randn((V, m), generator=g, device=dev) * (6 / m ** 0.5)
    head *= torch.exp(-4 * torch.arange(m, device=dev) / m)       # a spectrum that falls
    X = torch.randn((rows, n), generator=g, device=dev)

    # the uncompressed model's top logits
    teacher = torch.nn.functional.layer_norm(X @ W.t(), (m,)) @ head.t()
    t = torch.topk(teacher, top, dim=1)

    layer = Layer(W, k)
    X16 = torch.zeros((rows, lrc.lrc_packed_ld(n)), dtype=torch.float16, device=dev)
    X16[:, :n] = X
    exact = X[:1].double() @ W.double().t()
    err = [float((layer(X16[:1], c).double() - exact).norm() / exact.norm()) for c in (False, True)]
    print(f"4-bit layer {m} x {n}: eta {layer.eta:.4f}; one token off by {err[0]:.4f}, with rank {k} beside the codes "
          f"{err[1]:.4f}")

    repair = Repair(layer, factors(head, head_rank, "f32"), V, head_rank, t.values.contiguous(), t.indices, X16, tau=2.0)
    losses = [repair.step(2e-2) for _ in range(steps)]
    print(f"distillation loss over {rows} rows of {V} logits: {losses[0]:.4f} -> {losses[-1]:.4f} in {steps} steps of "
          "gamma and beta")
    return err, losses


if __name__ == "__main__":
    main()
