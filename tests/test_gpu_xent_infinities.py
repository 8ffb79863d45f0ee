"""Infinities in x and w: a logit that is infinite other than by its class's bias is a NaN, whichever way it points and whichever kernel has the row."""
import math

import pytest
import torch

from test_gpu_xent import TYPES, backward, forward, make
from test_gpu_xent_exact import KERNELS

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("dtype, m, v, k", KERNELS)
def test_an_infinity_in_a_class_that_is_there(dtype, m, v, k, bias):
    """Every row's logit of that class is infinite or NaN: rows whose x has the one sign and the other there, and zero."""
    x, w, targets, b, grad = make(m, v, k, TYPES[dtype], seed=21, bias=bias)
    if bias:
        b[v // 3] = b[v - 1] = -math.inf  # (classes that are taken out, beside)
    x[:, 7] = torch.tensor([1.0, -1.0, 2.0, -0.5, 0.0], device="cuda").repeat(m // 5 + 1)[:m].to(x.dtype)
    if m > 1:
        targets[m // 2] = -1
    have = targets >= 0
    for value in (math.inf, -math.inf):
        for at in (0, v // 2, v - 2):
            bad = w.clone()
            bad[at, 7] = value
            loss, lse = forward(x, bad, targets, b)
            assert bool(lse.isnan().all()) and bool(loss[have].isnan().all()) and bool((loss[~have] == 0).all()), (value, at)
    dx, dw, dbias = backward(x, bad, targets, lse, grad, b)
    assert bool(dx[have].isnan().all()) and bool(dw.isnan().any())
    out = b == -math.inf if bias else torch.zeros(v, dtype=torch.bool, device="cuda")
    assert bool(dbias[~out].isnan().all())


@pytest.mark.parametrize("dtype, m, v, k", KERNELS)
def test_an_infinity_in_a_row(dtype, m, v, k):
    """The row's logits are infinities of one sign alone, and the other rows are what they are without."""
    x, w, targets, b, _ = make(m, v, k, TYPES[dtype], seed=22)
    w[:, 7] = w[:, 7].abs() + 0.125
    loss0, lse0 = forward(x, w, targets, b)
    for value in (math.inf, -math.inf):
        row = m // 2
        bad = x.clone()
        bad[row, 7] = value
        loss, lse = forward(bad, w, targets, b)
        rest = torch.arange(m, device="cuda") != row
        assert bool(lse[row].isnan()) and bool(loss[row].isnan()) and torch.equal(lse[rest], lse0[rest]) and torch.equal(loss[rest], loss0[rest]), value


@pytest.mark.parametrize("dtype, m, v, k", [s for s in KERNELS if s[0] != "f16"])
def test_a_logit_that_overflows(dtype, m, v, k):
    x, w, targets, _, _ = make(m, v, k, TYPES[dtype], seed=23, bias=False)
    x[:, 7] = 1e30
    for value in (1e30, -1e30):
        w[v // 2, 7] = value
        loss, lse = forward(x, w, targets)
        assert bool(lse.isnan().all()) and bool(loss.isnan().all()), value
