"""The 4-bit product of binary32 vectors whose entries are very small: the three
parts of an entry hold all of its 24 bits, down to the smallest number."""
import pytest
import torch

import layer_ref as R
from layer_ref import U

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("b", [4, 10, 21, 43])
@pytest.mark.parametrize("group,zeros", [(32, True), (128, False)])
def test_apply_binary32_of_small_entries(lrc, cuda, b, group, zeros):
    """One entry a vector, of every binary order down to 2^-149, against scales of
    2^40: the parts' products are exact, each of the three sums holds one, so what
    is rounded is three scalings and two additions, each within U of the result's
    magnitude (the parts have one sign): 5 U of it, 6 with the second order."""
    m, n = 40, 256
    gen = torch.Generator(device=cuda).manual_seed(b + group)
    codes = torch.randint(0, 16, (m, n), generator=gen, device=cuda)
    scales = torch.full((n // group, R.ld16(m)), float("nan"), device=cuda)
    scales[:, :m] = (1 + torch.rand((n // group, m), generator=gen, device=cuda)) * 2.0 ** 40
    z = torch.randint(0, 16, scales.shape, generator=gen, device=cuda).to(torch.uint8) if zeros else None
    Q = R.q4_pack(codes)
    values = R.q4_values(Q, scales, z, m, n, group)
    orders = list(range(-149, 30))
    for first in range(0, len(orders), b):
        X = torch.zeros((b, n), device=cuda)
        for v in range(b):
            e = orders[(first + v) % len(orders)]
            bits = (1 << 23) + int(torch.randint(0, 1 << 23, (1,), generator=gen, device=cuda))
            # (below 2^-126 fewer bits are left: a whole multiple of 2^-149)
            x = max(1, bits >> max(0, -126 - e)) * 2.0 ** (max(e, -126) - 23)
            X[v, (37 * v + first) % n] = x if v % 2 else -x
        Y = torch.empty((b, m), device=cuda)
        lrc.lrc_q4_apply(Q, scales, z, X, None, Y, m, n, b, group, "f32")
        want = X.double() @ values.t()
        R.within(Y, want, 6 * U * want.abs(), f"orders from {orders[first]}")
