"""Distillation at temperatures near the ends of binary32's range."""
import math

import pytest
import torch

import layer_ref as R
import paper_2607_12969_gb300 as lrc
from layer_ref import U
from test_abi import L                     # noqa: F401  (the fixture)

P, F32 = 4096, 1


def test_a_temperature_without_a_factor_is_refused(L):     # noqa: F811
    """log2(e) / tau has to be a binary32 number, not 1 / tau alone."""
    def both(tau):
        return (L.lrc_distill(P, P, P, None, P, P, P, 0, 9, 3, 9, 3, 9, tau, F32, F32, None),
                L.lrc_distill_grad(P, P, P, None, P, None, P, 0, 9, 3, 9, 3, 9, tau, F32, F32, None))

    assert both(3e-39) == (-1, -1) and both(4.2e-39) == (-1, -1)
    assert both(4.3e-39) == (0, 0) and both(3.4e38) == (0, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("tau,weight", [(1e-30, 1e20), (2.0 ** -80, 1.0), (2.0 ** 66, 2.0 ** -40), (1e25, 1e-30)])
def test_the_factor_of_a_loss_is_not_formed_alone(cuda, tau, weight):
    """tau^2 leaves binary32, the loss does not.  At a low temperature each softmax is
    its largest entry, and the loss tau w times the distance of that entry's logit
    from the row's largest (three roundings); at a high one both are uniform: tau^2 w
    log(V / K), of whose factor a sum of V terms and the logarithms are within
    (V / 256 + 60) U."""
    lrc.load()
    rows, V, K = 3, 700, 8
    gen = torch.Generator(device=cuda).manual_seed(1)
    z = torch.randn((rows, V), generator=gen, device=cuda)
    t = torch.randn((rows, K), generator=gen, device=cuda)
    idx = torch.stack([torch.randperm(V, generator=gen, device=cuda)[:K] for _ in range(rows)])
    w = torch.full((rows,), weight, device=cuda)
    loss = torch.empty(rows, device=cuda)
    lrc.lrc_distill(z, t, idx, w, loss, None, None, rows, V, K, V, K, V, tau, "f32", "f32")
    tau, weight = float(torch.tensor(tau)), float(torch.tensor(weight))
    if tau < 1:
        best = z.gather(1, idx.gather(1, t.argmax(1, keepdim=True)))[:, 0]
        want = tau * weight * (z.amax(1).double() - best.double())
    else:
        want = torch.full((rows,), tau * weight * tau * math.log(V / K), dtype=torch.float64, device=cuda)
    R.within(loss, want, ((V / 256 + 60) * 2 * U) * want.abs())
