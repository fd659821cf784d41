"""Distillation at temperatures near the ends of binary32's range."""
from test_abi import L                     # noqa: F401  (the fixture)

P, F32 = 4096, 1


def test_a_temperature_without_a_factor_is_refused(L):     # noqa: F811
    """log2(e) / tau has to be a binary32 number, not 1 / tau alone."""
    def both(tau):
        return (L.lrc_distill(P, P, P, None, P, P, P, 0, 9, 3, 9, 3, 9, tau, F32, F32, None),
                L.lrc_distill_grad(P, P, P, None, P, None, P, 0, 9, 3, 9, 3, 9, tau, F32, F32, None))

    assert both(3e-39) == (-1, -1) and both(4.2e-39) == (-1, -1)
    assert both(4.3e-39) == (0, 0) and both(3.4e38) == (0, 0)
