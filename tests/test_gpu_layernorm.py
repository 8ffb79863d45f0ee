"""Layer norm forward and backward against plain references in 64 bits."""
import numpy as np
import pytest
import torch

import mx_reference as ref
from mx_reference import HALF_ULP, TINY, TYPES, backward_bounds, f64, on_gpu, sum_steps

pytestmark = pytest.mark.gpu
EPS = 1e-5
ULP = HALF_ULP["f32"]


def _dq():
    import paper_2410_20046_amd as dq

    return dq


def _forward_bounds(x, gamma, beta, y, mean, rstd, dtype):
    """Of mean, rstd and y, from the roundings of the sums and of each step behind them (first order, doubled)."""
    n = x.shape[1]
    s = sum_steps(n)
    size = np.abs(x).mean(1)
    b_mean = (s + 2) * ULP * size
    # (x - mean) is off by the mean's error and its own rounding; the squares' sum by twice that, relative
    d = np.abs(x - mean[:, None])
    off_d = b_mean[:, None] + ULP * d
    off_var = (2 * d * off_d).mean(1) + off_d.max(1) ** 2 + (s + 4) * ULP * (d * d).mean(1)
    b_rstd = 0.5 * off_var * rstd ** 3 + 4 * ULP * rstd
    xh = d * rstd[:, None]
    b_y = (off_d * rstd[:, None] + d * b_rstd[:, None] + 3 * ULP * xh) * np.abs(gamma) + ULP * np.abs(beta) + ULP * np.abs(y)
    return 2 * b_mean + 1e-45, 2 * b_rstd, 2 * b_y + 1.01 * HALF_ULP[dtype] * np.abs(y) + TINY[dtype]


def _gain(rng, C, kind):
    if kind == "none":
        return None, None, 1.0, 0.0
    g, b = (1 + 0.4 * rng.standard_normal(C)).astype(np.float32), rng.standard_normal(C).astype(np.float32)
    return torch.from_numpy(g).cuda(), torch.from_numpy(b).cuda(), g.astype(np.float64), b.astype(np.float64)


# every way a row is laid over threads, and both sides of each limit
SHAPES = [(1, 1), (5, 2), (3, 7), (130, 13), (17, 128), (16, 129), (1000, 64), (33, 512), (9, 513), (6, 1024), (7, 1025), (4, 2048), (5, 2049),
          (3, 4097), (2, 8191), (3, 8193), (2, 16384), (3, 16385), (2, 50001), (300, 700), (290, 1500), (280, 2500), (270, 6000)]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_forward(shape, dtype):
    dq = _dq()
    R, C = shape
    rng = np.random.default_rng(R + 10 * C)
    print("norm", shape, dtype, flush=True)
    for stride, offset, kind in ((C, 0, "both"), (C + 3, 1, "none"), ((C + 7) // 8 * 8, 0, "both")):
        x = on_gpu(rng.standard_normal((R, C)) * np.exp2(rng.integers(-4, 5, (R, 1))) + 3.0, TYPES[dtype], stride, offset)
        g, b, gv, bv = _gain(rng, C, kind)
        y = on_gpu(np.zeros((R, C)), TYPES[dtype], stride + 1, 1)
        around = y._base.clone()
        mean, rstd = torch.empty(R, device="cuda"), torch.empty(R, device="cuda")
        q = dq.MxMatrix(R, C, "cuda")
        q.codes.fill_(0xA5), q.scales.fill_(0x5A)
        dq.dqrm_layernorm_fwd(x, g, b, EPS, y=y, mean=mean, rstd=rstd, q=q)
        want, m, r = ref.norm(f64(x), gv, bv, EPS)
        b_mean, b_rstd, b_y = _forward_bounds(f64(x), gv, bv, want, m, r, dtype)
        assert np.all(np.abs(f64(mean) - m) <= b_mean)
        assert np.all(np.abs(f64(rstd) - r) <= b_rstd)
        assert np.all(np.abs(f64(y) - want) <= b_y)
        # each output alone is the same
        y2 = torch.empty_like(y)
        dq.dqrm_layernorm_fwd(x, g, b, EPS, y=y2)
        assert torch.equal(y2, y)
        q2 = dq.MxMatrix(R, C, "cuda")
        dq.dqrm_layernorm_fwd(x, g, b, EPS, q=q2)
        assert torch.equal(q2.codes, q.codes) and torch.equal(q2.scales, q.scales)
        if dtype == "f32":  # y as it was quantised
            code, scale = ref.quantise(f64(y))
            np.testing.assert_array_equal(q.scales.cpu().numpy(), scale)
            np.testing.assert_array_equal(q.codes.cpu().numpy(), ref.pack(code))
        # in place
        xin = x.clone() if stride == C else on_gpu(f64(x), TYPES[dtype], stride, offset)
        dq.dqrm_layernorm_fwd(xin, g, b, EPS, y=xin)
        assert torch.equal(xin, y)
        y.fill_(0.0)
        assert torch.equal(y._base.nan_to_num(7.0), around.nan_to_num(7.0))


@pytest.mark.parametrize("cols", [100, 250, 384, 500, 1024, 1500, 2048, 2500, 4096, 5001, 8191, 10001, 16384])
def test_many_values_of_16_bits(cols):
    """The ways that a row is laid over threads where there are many values; the plain form in 64 bits on the GPU."""
    dq = _dq()
    dtype = "bf16" if cols % 2 else "f16"
    R = (1 << 22) // cols + 5
    print("norm of many values", (R, cols), dtype, flush=True)
    gen = torch.Generator("cuda").manual_seed(cols)
    rand = lambda *s: torch.randn(s, device="cuda", generator=gen)
    x, dy = (rand(R, cols) * 2 + 1).to(TYPES[dtype]), rand(R, cols).to(TYPES[dtype])
    g, b = 1 + 0.4 * rand(cols), rand(cols)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd, dgamma, dbeta = torch.empty(R, device="cuda"), torch.empty(R, device="cuda"), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    dq.dqrm_layernorm_fwd(x, g, b, EPS, y=y, mean=mean, rstd=rstd)
    ws = torch.full((dq.dqrm_layernorm_bwd_workspace_bytes(R, cols),), 0xFF, dtype=torch.uint8, device="cuda")
    dq.dqrm_layernorm_bwd(dy, x, mean, rstd, g, dx, dgamma, dbeta, ws)
    # some of the rows, the last ones among them, against the bounds of each value
    at = torch.cat([torch.arange(0, R, max(R // 40, 1)), torch.arange(R - 8, R)]).cuda()
    xv, dyv, gv = f64(x[at]), f64(dy[at]), f64(g)
    want, m, r = ref.norm(xv, gv, f64(b), EPS)
    b_mean, b_rstd, b_y = _forward_bounds(xv, gv, f64(b), want, m, r, dtype)
    assert np.all(np.abs(f64(mean[at]) - m) <= b_mean) and np.all(np.abs(f64(rstd[at]) - r) <= b_rstd) and np.all(np.abs(f64(y[at]) - want) <= b_y)
    wdx, _, _ = ref.norm_backward(dyv, xv, f64(mean[at]), f64(rstd[at]), gv)
    b_dx, _, _ = backward_bounds(dyv, xv, f64(mean[at]), f64(rstd[at]), gv, wdx, dtype, 0)
    assert np.all(np.abs(f64(dx[at]) - wdx) <= b_dx)
    # every row is in the sums
    xh = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    chain = min(R, 64) + R / 64 + 64
    for got, terms in ((dgamma, dy.double() * xh), (dbeta, dy.double())):
        assert bool(((got.double() - terms.sum(0)).abs() <= 1.01 * (chain + 3) * ULP * terms.abs().sum(0) + 1e-45).all())


@pytest.mark.parametrize("cols", [5, 200, 3000, 20000])
def test_rows_of_one_value_and_rows_that_are_not_finite(cols):
    dq = _dq()
    x = np.random.default_rng(0).standard_normal((6, cols)).astype(np.float32)
    x[0] = 0.0
    x[1] = 1234.5678
    x[2, cols // 2] = np.nan
    x[4, cols - 1] = np.inf
    xt = on_gpu(x, torch.float32, cols + 1, 1)
    y, mean, rstd, q = torch.empty((6, cols), device="cuda"), torch.empty(6, device="cuda"), torch.empty(6, device="cuda"), dq.MxMatrix(6, cols, "cuda")
    dq.dqrm_layernorm_fwd(xt, None, None, EPS, y=y, mean=mean, rstd=rstd, q=q)
    y, mean, rstd = f64(y), f64(mean), f64(rstd)
    assert np.all(y[0] == 0) and mean[0] == 0
    # the mean of equal values is off by the sum's roundings: y by that over sqrt(eps)
    assert np.all(np.abs(y[1]) <= 2 * sum_steps(cols) * ULP * 1235 / np.sqrt(EPS))
    for r in (2, 4):
        assert np.isnan(y[r]).all()
        assert (q.scales[r].cpu().numpy()[: -(-cols // 32)] == 255).all()
    for r in (3, 5):
        assert np.isfinite(y[r]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shape", SHAPES + [(5000, 40), (2100, 300), (3, 70000)])
def test_backward(shape, dtype):
    dq = _dq()
    R, C = shape
    rng = np.random.default_rng(R + 10 * C)
    print("norm backward", shape, dtype, flush=True)
    for stride, offset, kind in ((C, 0, "both"), (C + 3, 1, "none"), ((C + 7) // 8 * 8, 0, "both")):
        x = on_gpu(rng.standard_normal((R, C)) * 2 + 1, TYPES[dtype], stride, offset)
        dyv = rng.standard_normal((R, C)) * np.exp2(rng.integers(-6, 3, (R, 1)))
        dyv[:: 4] = 0.0  # rows without a gradient
        dy = on_gpu(dyv, TYPES[dtype], stride + 1, 1)
        g, _, gv, _ = _gain(rng, C, kind)
        mv = f64(x).mean(1)
        mean = torch.from_numpy(mv).float().cuda()
        rstd = torch.from_numpy(1 / np.sqrt(f64(x).var(1) + EPS)).float().cuda()
        dx = on_gpu(np.zeros((R, C)), TYPES[dtype], stride + 2, 1)
        around = dx._base.clone()
        dgamma, dbeta = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
        ws = torch.full((dq.dqrm_layernorm_bwd_workspace_bytes(R, C),), 0xFF, dtype=torch.uint8, device="cuda")
        dq.dqrm_layernorm_bwd(dy, x, mean, rstd, g, dx, dgamma, dbeta, ws)
        wdx, wdg, wdb = ref.norm_backward(f64(dy), f64(x), f64(mean), f64(rstd), gv)
        # a column's sums: the rows of a slice in turn, slices in turn, at most one slice to 32 rows of long rows
        chain = min(R, 64) + R / 64 + 64
        b_dx, b_dg, b_db = backward_bounds(f64(dy), f64(x), f64(mean), f64(rstd), gv, wdx, dtype, chain)
        assert np.all(np.abs(f64(dx) - wdx) <= b_dx)
        assert np.all(np.abs(f64(dgamma) - wdg) <= b_dg)
        assert np.all(np.abs(f64(dbeta) - wdb) <= b_db)
        # parts of the outputs, and in place over either input
        dx2, dg2, db2 = torch.empty_like(dx), torch.empty_like(dgamma), torch.empty_like(dbeta)
        dq.dqrm_layernorm_bwd(dy, x, mean, rstd, g, dx2)
        dq.dqrm_layernorm_bwd(dy, x, mean, rstd, g, None, dg2, db2, ws)
        assert torch.equal(dx2, dx) and torch.equal(dg2, dgamma) and torch.equal(db2, dbeta)
        for which in (0, 1):
            a = [on_gpu(f64(dy), TYPES[dtype], stride + 1, 1), on_gpu(f64(x), TYPES[dtype], stride, offset)]
            dq.dqrm_layernorm_bwd(a[0], a[1], mean, rstd, g, a[which], dg2, db2, ws)
            assert torch.equal(a[which], dx) and torch.equal(dg2, dgamma) and torch.equal(db2, dbeta)
        dx.fill_(0.0)
        assert torch.equal(dx._base.nan_to_num(7.0), around.nan_to_num(7.0))


def test_no_rows():
    dq = _dq()
    x, v = torch.empty((0, 9), device="cuda"), torch.empty(0, device="cuda")
    dq.dqrm_layernorm_fwd(x, None, None, EPS, y=x, mean=v, rstd=v)
    dg, db = torch.full((9,), 3.0, device="cuda"), torch.full((9,), 3.0, device="cuda")
    dq.dqrm_layernorm_bwd(x, x, v, v, None, x, dg, db)
    assert torch.equal(dg, torch.zeros_like(dg)) and torch.equal(db, torch.zeros_like(db))


@pytest.mark.parametrize("cols", [3, 70, 600])
def test_backward_against_differences(cols):
    """Central differences, in 64 bits, of the loss sum(dy y): within the difference's own error of step^2 and the kernel's."""
    dq = _dq()
    R = 7
    rng = np.random.default_rng(cols)
    x, dy = rng.standard_normal((R, cols)), rng.standard_normal((R, cols))
    gamma, beta = 1 + 0.3 * rng.standard_normal(cols), rng.standard_normal(cols)
    put = lambda a: torch.from_numpy(np.asarray(a)).float().cuda()  # noqa: E731
    x, dy, gamma, beta = (a.astype(np.float32).astype(np.float64) for a in (x, dy, gamma, beta))
    _, m, r = ref.norm(x, gamma, beta, EPS)
    dx, dg, db = torch.empty((R, cols), device="cuda"), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    ws = torch.empty(dq.dqrm_layernorm_bwd_workspace_bytes(R, cols), dtype=torch.uint8, device="cuda")
    dq.dqrm_layernorm_bwd(put(dy), put(x), put(m), put(r), put(gamma), dx, dg, db, ws)
    loss = lambda: float((dy * ref.norm(x, gamma, beta, EPS)[0]).sum())  # noqa: E731
    h = 1e-4
    for arr, grad in ((x, f64(dx)), (gamma, f64(dg)), (beta, f64(db))):
        for _ in range(12):
            at = tuple(int(rng.integers(0, s)) for s in arr.shape)
            old = arr[at]
            arr[at] = old + h
            up = loss()
            arr[at] = old - h
            down = loss()
            arr[at] = old
            # third derivatives of y in x are of the order of rstd^3 (|y| + ...): h^2 of them, with room
            assert abs((up - down) / (2 * h) - grad[at]) <= 1e-5 * (1 + np.abs(grad).max()) + 100 * h * h * r.max() ** 3 * np.abs(dy).max()
