"""On the CPU: what tests/test_gpu_xent_planes.py allows is less than what any one lost plane product makes."""
import pytest
import torch

from plane_reference import PAIRS, PRODUCT, U, lse_and_bound, planes, product, values


def test_planes_are_the_values():
    v = values((100, 100), 1)
    p = planes(v)
    assert bool((p[0] + p[1] + p[2] == v.double()).all()) and all(bool((q > 0).all()) for q in p)


@pytest.mark.parametrize("v", [300, 33000])
@pytest.mark.parametrize("lost", [(p,) for p in PAIRS] + [((1, 0), (1, 1)), ((0, 2), (1, 1), (2, 0)), ()])
def test_a_lost_product_is_seen(lost, v):
    a, b, scale = values((20, 1), 2), values((1, v), 3), 64.0
    exact, some = a.double() * b.double(), product(a, b, [p for p in PAIRS if p not in lost])
    lse, off = lse_and_bound(some * scale, exact * scale)
    far = (lse - torch.logsumexp(exact * scale, 1)).abs()
    # gradients are single products too: with d's three roundings, the unit's and the scale's, and the result's
    gone = (some - exact).abs() / exact / (PRODUCT + 7 * U)
    if lost:
        assert bool((far > 2 * off).all()) and bool((gone > 2).all())
    else:
        assert bool((far < 0.25 * off).all()) and bool((gone < 0.25).all())
