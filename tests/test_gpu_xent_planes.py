"""The loss of fp32 operands whose logits and gradients are single products, of which each of the six plane products counts."""
import pytest
import torch

from plane_reference import PRODUCT, U, lse_and_bound, values
from test_gpu_xent import backward, forward
from test_gpu_xent_exact import KERNELS

pytestmark = pytest.mark.gpu

SHAPES = [s[1:] for s in KERNELS if s[0] == "f32"] + [(300, 1000, 200), (8, 300, 2100)]


@pytest.mark.parametrize("m, v, k", SHAPES)
def test_each_plane_product_of_the_logits_and_of_both_gradients(m, v, k):
    scale = 64.0
    rows = torch.arange(m)
    place = rows * 7 % k
    x = torch.zeros(m, k)
    x[rows, place] = values((m,), 4)
    w = values((v, k), 5)
    exact = x[rows, place].double()[:, None] * w[:, place].t().double() * scale
    targets = rows * (v // m) % v
    x, w, targets, exact, place, rows = (t.cuda() for t in (x, w, targets, exact, place, rows))
    _, lse = forward(x, w, targets, None, scale)
    want, off = lse_and_bound(exact, exact)
    assert bool(((lse.double() - want).abs() <= off).all()), float(((lse.double() - want).abs() / off).max())
    # an lse far above the logits: all probabilities are 0, and d is -grad at the target; grad in units of the largest, 1
    grad = values((m,), 6).cuda() / 2
    grad[0] = 1
    dx, dw, _ = backward(x, w, targets, torch.full((m,), 1e4, device="cuda"), grad, None, scale)
    least = PRODUCT + 7 * U
    want = -scale * grad.double()[:, None] * w[targets].double()
    assert bool(((dx.double() - want).abs() <= least * want.abs()).all()), float(((dx.double() - want).abs() / want.abs()).max() / least)
    want = torch.zeros(v, k, dtype=torch.float64, device="cuda")
    want[targets, place] = -scale * grad.double() * x[rows, place].double()
    assert bool(((dw.double() - want).abs() <= least * want.abs()).all()), float(((dw.double() - want).abs().max() / least / scale))
