"""Infinities in x and w: a logit that is infinite other than by its class's bias is a NaN, whichever way it points and whichever kernel has the row."""
import math

import pytest
import torch

from test_gpu_xent import TYPES, backward, forward, make
from test_gpu_xent_exact import KERNELS
from xent_reference import gradients_and_bounds, near

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


@pytest.mark.parametrize("dtype, m, v, k", KERNELS)
def test_a_target_that_is_taken_out(dtype, m, v, k):
    """The loss is infinite.  d is -grad at the target, in dw and dbias too; dx leaves aside what w holds there: it is the gradient of lse."""
    x, w, targets, b, grad = make(m, v, k, TYPES[dtype], seed=24)
    targets = targets % 5 + torch.arange(m, device="cuda") % 2 * (v // 2)  # (some rows' alone)
    out = torch.zeros(v, dtype=torch.bool, device="cuda")
    out[targets[::2]] = True
    b[out] = -math.inf
    r = gradients_and_bounds(x, w, targets, b, 1.0, grad)
    bad = w.clone()
    bad[out] = math.nan
    loss, lse = forward(x, bad, targets, b)
    near(loss, r["loss"], r["loss_off"], "loss")
    near(lse, r["lse"], r["lse_off"], "lse")
    assert bool((loss.isinf() == out[targets]).all())
    dx, dw, dbias = backward(x, bad, targets, lse, grad, b)
    near(dx, *r["dx"], "dx")
    near(dw, *r["dw"], "dw")
    near(dbias, *r["dbias"], "dbias")
    # of such a class there is nothing but its targets' part
    of = torch.zeros(v, dtype=torch.float64, device="cuda").index_add_(0, targets, grad.double())
    assert bool((of[out] > 0).any()) and bool(((dbias.double() + of)[out].abs() <= (m + 8) * 2.0 ** -24 * of[out]).all())


@pytest.mark.parametrize("dtype, m, v, k", KERNELS)
def test_a_bias_of_the_lowest_value(dtype, m, v, k):
    """A class whose bias is float's lowest value is taken out as one with -infinity: its logit in powers of two is -infinity, whatever w holds."""
    x, w, targets, b, grad = make(m, v, k, TYPES[dtype], seed=25)
    out = torch.arange(v, device="cuda") % 3 == 1
    w[out] = math.nan
    targets = torch.where(torch.arange(m, device="cuda") % 4 == 0, targets // 3 * 3 + 1, targets).clamp(max=v - 2)  # (some rows' among them)
    got = []
    for value in (-math.inf, torch.finfo(torch.float32).min):
        b[out] = value
        loss, lse = forward(x, w, targets, b)
        got.append((loss, lse, *backward(x, w, targets, lse, grad, b)))
    assert all(torch.equal(p, q) for p, q in zip(*got)) and bool(lse.isfinite().all()) and not any(bool(t.isnan().any()) for t in got[0])
    b[:] = torch.finfo(torch.float32).min  # no class left
    loss, lse = forward(x, w, targets, b)
    assert bool((lse == -math.inf).all()) and bool((loss == math.inf).all())
    for t in backward(x, w, targets, lse, grad, b):
        assert bool((t == 0).all())
