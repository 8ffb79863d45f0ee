"""Products, linear layers and norms at shapes that every kernel of the library for them is launched at (test_mxfp4_coverage.py checks on
the CPU that they are), in each type, with bias, ReLU and rows that start anywhere; references in 64 bits, on the GPU where they are large."""
import numpy as np
import pytest
import torch

import mx_reference as ref
import test_gpu_layernorm as norms
from mx_reference import HALF_ULP, TINY, TYPES, backward_bounds, f64

pytestmark = pytest.mark.gpu

#: (m, n, k): tiles of 64, of 128 one and two to a CU and of 256, k whole and in slices, with odd numbers of stages of 256 and without; few
#: rows in groups of 16, 32 and 64 with one strip of W to a workgroup and with two
PRODUCTS = [(1500, 700, 900), (174, 104, 5194), (1797, 1517, 2059), (2041, 2039, 8192), (1045, 590, 12571), (2100, 1999, 1500), (4100, 4097, 700),
            (973, 1391, 17715), (4096, 4096, 1100), (2473, 3268, 2056), (1601, 1689, 28379), (1, 512, 367), (16, 16500, 300), (30, 5000, 200),
            (20, 16500, 300), (60, 300, 3000), (50, 8300, 1100)]
#: rows that the product quantises itself; k even
LINEAR = [(1, 512, 368), (1, 16400, 368), (2, 16500, 300), (3, 16401, 8), (4, 16390, 1000), (4, 300, 2000), (2, 40, 4096)]
#: 16-bit matrices of many values: bfloat16 where odd, half where even
MANY = [249, 383, 1499, 2047, 2499, 5002, 10002]
#: (rows, columns, row stride) past 2^31 values
LARGE = [(150000, 16384, 16384), (70000, 8191, 40000), (35000, 70001, 70001)]


def _dq():
    import paper_2410_20046_amd as dq

    return dq


def _space(n):
    return torch.full((max(int(n), 256),), 0xFF, dtype=torch.uint8, device="cuda")


def _room(rows, cols, stride, offset, dtype):
    """A matrix in memory that is NaN, the memory, and a check that nothing but the matrix was written."""
    memory = torch.full((offset + rows * stride + 16,), float("nan"), dtype=dtype, device="cuda")
    out = memory[offset:offset + rows * stride].view(rows, stride)[:, :cols]

    def untouched():
        keep = out.clone()
        out.fill_(float("nan"))
        ok = bool(memory.isnan().all())
        out.copy_(keep)
        return ok

    return out, untouched


def _held(values):
    """A matrix in MXFP4 and what it stands for, in 64 bits, both on the GPU."""
    dq = _dq()
    q = dq.MxMatrix(*values.shape, "cuda")
    dq.dqrm_mxfp4_quant(values, q)
    out = torch.empty_like(values)
    dq.dqrm_mxfp4_dequant(q, out)
    return q, out.double()


def _check(out, full, size, k, relu, dtype):
    """As in test_gpu_mxfp4: sums of 64 products at a time that lose two units in the last place, partial sums in turn, one rounding."""
    want = full.clamp_min(0.0) if relu else full
    bound = (k / 64 + 40) * 2.0 ** -22 * size + 1.01 * HALF_ULP[dtype] * want.abs() + TINY[dtype]
    off = (out.double() - want).abs()
    assert bool((off <= bound).all()), (tuple(out.shape), dtype, float(off.max()))


@pytest.mark.parametrize("shape", PRODUCTS)
def test_product_in_each_type(shape):
    dq = _dq()
    m, n, k = shape
    gen = torch.Generator("cuda").manual_seed(m + n + k)
    rand = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
    # scales from row to row, small enough for half precision's outputs
    a, av = _held(rand(m, k) * torch.exp2(torch.randint(-4, 1, (m, 1), device="cuda", generator=gen).float()))
    b, bv = _held(rand(n, k) * torch.exp2(torch.randint(-4, 1, (n, 1), device="cuda", generator=gen).float()))
    bias = rand(n)
    full, size = av @ bv.t().contiguous(), av.abs() @ bv.abs().t().contiguous()
    ws = _space(dq.dqrm_mxfp4_matmul_workspace_bytes(m, n, k))
    for dtype in TYPES:
        # rows from odd places on; rows of whole lines
        for stride, offset, with_bias, relu in ((n + 3, 1, True, True), ((n + 63) // 64 * 64, 0, False, False), (n, 0, True, False)):
            print("product", shape, dtype, stride, offset, flush=True)
            out, untouched = _room(m, n, stride, offset, TYPES[dtype])
            dq.dqrm_mxfp4_matmul(a, b, out, bias=bias if with_bias else None, relu=relu, workspace=ws)
            add = bias.double() if with_bias else torch.zeros(n, dtype=torch.float64, device="cuda")
            _check(out, full + add, size + add.abs(), k, relu, dtype)
            assert untouched()


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("shape", LINEAR)
def test_linear_of_rows_that_the_product_quantises(shape, norm):
    """Behind the norm, rows of which half is 2^e and half -2^e: mean 0 and deviation 2^e without any rounding (eps = 0), so that a value's
    code is the same whatever the order of the sums."""
    dq = _dq()
    m, n, k = shape
    rng = np.random.default_rng(m + n + k)
    gen = torch.Generator("cuda").manual_seed(m + n + k)
    w, wv = _held(torch.randn((n, k), device="cuda", generator=gen) / k ** 0.5)
    bias = torch.randn(n, device="cuda", generator=gen)
    ws = _space(dq.dqrm_mxfp4_linear_workspace_bytes(m, n, k))
    gamma, beta = rng.integers(-24, 25, k) / 8.0, rng.integers(-8, 9, k) / 8.0
    for dtype in TYPES:
        for stride, offset, relu in ((k, 0, True), (k + 5, 3, False)):
            print("linear", shape, norm, dtype, stride, flush=True)
            if norm:
                values = np.stack([rng.permutation(np.repeat([1.0, -1.0], k // 2)) for _ in range(m)])
                x = values * np.exp2(rng.integers(-3, 4, (m, 1)))
                options = dict(gamma=torch.from_numpy(gamma).float().cuda(), beta=torch.from_numpy(beta).float().cuda(), eps=0.0)
                given = values * gamma + beta
            else:
                x = torch.from_numpy(rng.standard_normal((m, k)) * np.exp2(rng.integers(-4, 2, (m, 1)))).to(TYPES[dtype]).double().numpy()
                options, given = {}, x
            held, _ = _room(m, k, stride, offset, TYPES[dtype])
            held.copy_(torch.from_numpy(x))
            out, untouched = _room(m, n, n + 3, 1, TYPES[dtype])
            dq.dqrm_mxfp4_linear(held, w, out, bias=bias, relu=relu, workspace=ws, **options)
            xv = torch.from_numpy(ref.quantised_values(given)).cuda()
            _check(out, xv @ wv.t().contiguous() + bias.double(), xv.abs() @ wv.abs().t().contiguous() + bias.double().abs(), k, relu, dtype)
            assert untouched()


@pytest.mark.parametrize("cols", MANY)
def test_norms_of_many_values(cols):
    norms.test_many_values_of_16_bits(cols)


@pytest.mark.parametrize("rows, cols, stride", LARGE)
def test_norms_past_32_bits(rows, cols, stride):
    """Every output of matrices whose last values are past 2^31: some rows against the bounds of each value, and all rows' sums."""
    dq = _dq()
    print("norms", rows, cols, stride, flush=True)
    dtype, eps = "bf16", 1e-5
    gen = torch.Generator("cuda").manual_seed(cols)
    x, dy, y = (torch.empty((rows, stride), dtype=torch.bfloat16, device="cuda")[:, :cols] for _ in range(3))
    for r0 in range(0, rows, 8192):
        x[r0:r0 + 8192].copy_(torch.randn(x[r0:r0 + 8192].shape, device="cuda", generator=gen) + 0.5)
        dy[r0:r0 + 8192].copy_(torch.randn(x[r0:r0 + 8192].shape, device="cuda", generator=gen))
    gamma, beta = 1 + 0.4 * torch.randn(cols, device="cuda", generator=gen), torch.randn(cols, device="cuda", generator=gen)
    mean, rstd, dgamma, dbeta = (torch.empty(s, device="cuda") for s in (rows, rows, cols, cols))
    q = dq.MxMatrix(rows, cols, "cuda")
    dq.dqrm_layernorm_fwd(x, gamma, beta, eps, y=y, mean=mean, rstd=rstd, q=q)
    edge = (1 << 31) // stride  # the row that value 2^31 is in
    few = sorted({r for r in (0, 1, 32767, 32768, 65535, 65536, edge - 1, edge, edge + 1, rows - 2, rows - 1) if r < rows})
    xv, gv, bv = f64(x[few]), f64(gamma), f64(beta)
    want, m, r = ref.norm(xv, gv, bv, eps)
    b_mean, b_rstd, b_y = norms._forward_bounds(xv, gv, bv, want, m, r, dtype)
    assert np.all(np.abs(f64(mean[few]) - m) <= b_mean) and np.all(np.abs(f64(rstd[few]) - r) <= b_rstd) and np.all(np.abs(f64(y[few]) - want) <= b_y)
    # the codes, from y before its rounding: within a rounding of it and a step between codes
    held = dq.MxMatrix(len(few), cols, codes=q.codes[few].contiguous(), scales=q.scales[few].contiguous())
    back = torch.empty((len(few), cols), device="cuda")
    dq.dqrm_mxfp4_dequant(held, back)
    block = np.abs(np.pad(want, ((0, 0), (0, -cols % 32)))).reshape(len(few), -1, 32).max(-1).repeat(32, 1)[:, :cols]
    assert np.all(np.abs(f64(back) - want) <= block / 4 * 1.01)
    ws = _space(dq.dqrm_layernorm_bwd_workspace_bytes(rows, cols))
    dx = y
    dq.dqrm_layernorm_bwd(dy, x, mean, rstd, gamma, dx, dgamma, dbeta, ws)
    dyv, mv, rv = f64(dy[few]), f64(mean[few]), f64(rstd[few])
    wdx, _, _ = ref.norm_backward(dyv, xv, mv, rv, gv)
    assert np.all(np.abs(f64(dx[few]) - wdx) <= backward_bounds(dyv, xv, mv, rv, gv, wdx, dtype, 0)[0])
    sums = torch.zeros((4, cols), dtype=torch.float64, device="cuda")
    for r0 in range(0, rows, 4096):
        d = dy[r0:r0 + 4096].double()
        t = d * ((x[r0:r0 + 4096].double() - mean[r0:r0 + 4096, None].double()) * rstd[r0:r0 + 4096, None].double())
        for i, v in enumerate((t, t.abs(), d, d.abs())):
            sums[i] += v.sum(0)
    chain = min(rows, 64) + rows / 64 + 64
    assert bool(((dgamma.double() - sums[0]).abs() <= 1.01 * (chain + 3) * HALF_ULP["f32"] * sums[1]).all())
    assert bool(((dbeta.double() - sums[2]).abs() <= 1.01 * chain * HALF_ULP["f32"] * sums[3]).all())
