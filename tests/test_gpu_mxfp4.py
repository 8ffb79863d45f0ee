"""MXFP4 quantisation, dequantisation and products against plain references in 64 bits."""
import numpy as np
import pytest
import torch

import mx_reference as ref
from mx_reference import HALF_ULP, TINY, TYPES, backward_bounds, f64, on_gpu

pytestmark = pytest.mark.gpu


def _dq():
    import paper_2410_20046_amd as dq

    return dq


def _said(*what):
    print(*what, flush=True)


def _inputs(rng, R, C, hard=True):
    """Values of every size a block meets: blocks of zeros, midpoints between codes, subnormals, the largest numbers."""
    x = rng.standard_normal((R, C)) * np.exp2(rng.integers(-20, 20, (R, 1)))
    if hard:
        P = ref.pad128(C)
        v = np.zeros((R, P))
        v[:, :C] = x
        b = v.reshape(R, -1, 32)
        kind = rng.integers(0, 10, b.shape[:2])
        b[kind == 0] = 0.0
        mids = rng.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 7.9375, 4.0], b.shape) * rng.choice([-1, 1], b.shape)
        b[kind == 1] = (mids * np.exp2(rng.integers(-12, 10, (*b.shape[:2], 1))))[kind == 1]
        b[kind == 2] *= 2.0 ** -9 * rng.integers(0, 2, b.shape)[kind == 2]
        x = v[:, :C]
    return x


def _codes(q):
    return q.codes.cpu().numpy(), q.scales.cpu().numpy()


SHAPES = [(1, 1), (1, 13), (3, 31), (2, 32), (5, 33), (7, 127), (4, 128), (33, 129), (128, 415), (129, 367), (300, 64), (257, 513), (1, 5000), (2000, 1)]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_quantise_both_ways_and_back(shape, dtype):
    dq = _dq()
    R, C = shape
    rng = np.random.default_rng(R * 1000 + C)
    _said("quantise", shape, dtype)
    for stride, offset in ((C, 0), (C + 3, 1), ((C + 63) // 64 * 64, 0)):
        x = on_gpu(_inputs(rng, R, C), TYPES[dtype], stride, offset)
        q, qt = dq.MxMatrix(R, C, "cuda"), dq.MxMatrix(C, R, "cuda")
        alone, alone_t = dq.MxMatrix(R, C, "cuda"), dq.MxMatrix(C, R, "cuda")
        for m in (q, qt, alone, alone_t):
            m.codes.fill_(0xA5), m.scales.fill_(0x5A)
        dq.dqrm_mxfp4_quant(x, q, qt)
        dq.dqrm_mxfp4_quant(x, alone)
        dq.dqrm_mxfp4_quant(x, None, alone_t)
        for got, other, want in ((q, alone, f64(x)), (qt, alone_t, f64(x).T)):
            code, scale = ref.quantise(want)
            for m in (got, other):
                c, s = _codes(m)
                np.testing.assert_array_equal(s, scale)
                np.testing.assert_array_equal(c, ref.pack(code))
            for out_type in TYPES:
                out = on_gpu(np.zeros(want.shape), TYPES[out_type], want.shape[1] + 5, 3)
                around = out._base.clone()
                dq.dqrm_mxfp4_dequant(got, out)
                v = torch.from_numpy(ref.values(ref.pack(code), scale, want.shape[1])).to(torch.float32).to(TYPES[out_type])
                assert torch.allclose(out.cpu(), v, rtol=0, atol=0, equal_nan=True)
                out.fill_(0.0)
                assert torch.equal(out._base.nan_to_num(7.0), around.nan_to_num(7.0))  # nothing beside the matrix is written


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_blocks_with_infinities_and_nans_are_nan_and_the_others_are_not(dtype):
    dq = _dq()
    x = np.random.default_rng(3).standard_normal((130, 200))
    x[3, 40], x[70, 5], x[129, 199], x[4, 64] = np.nan, np.inf, -np.inf, -np.nan
    x = on_gpu(x, TYPES[dtype])
    q, qt = dq.MxMatrix(130, 200, "cuda"), dq.MxMatrix(200, 130, "cuda")
    dq.dqrm_mxfp4_quant(x, q, qt)
    for m, want in ((q, f64(x)), (qt, f64(x).T)):
        code, scale = ref.quantise(want)
        assert (scale == 255).sum() == 4
        c, s = _codes(m)
        np.testing.assert_array_equal(s, scale)
        np.testing.assert_array_equal(c, ref.pack(code))
        out = torch.empty(want.shape, device="cuda")
        dq.dqrm_mxfp4_dequant(m, out)
        np.testing.assert_array_equal(f64(out), ref.values(ref.pack(code), scale, want.shape[1]))


def test_blocks_of_the_smallest_and_largest_numbers():
    dq = _dq()
    top = np.float32(3.4028234663852886e38)
    rows = [[1e-45, 0, -1e-45], [1e-39, 3e-39, -7e-39], [2.0 ** -126, 2.0 ** -128, 2.0 ** -129 * 1.5], [top, -top, top / 3],
            [2.0 ** -127, 2.0 ** -130, 1.5 * 2.0 ** -129], [2.0 ** -124, 2.0 ** -125, 2.0 ** -129], [-0.0, 0.0, -0.0]]
    x = on_gpu(np.array(rows, np.float32), torch.float32)
    q = dq.MxMatrix(len(rows), 3, "cuda")
    dq.dqrm_mxfp4_quant(x, q)
    code, scale = ref.quantise(f64(x))
    c, s = _codes(q)
    np.testing.assert_array_equal(s, scale)
    np.testing.assert_array_equal(c, ref.pack(code))
    out = torch.empty(x.shape, device="cuda")
    dq.dqrm_mxfp4_dequant(q, out)
    np.testing.assert_array_equal(f64(out), ref.values(ref.pack(code), scale, 3))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shape", [(1, 1), (37, 70), (128, 128), (1000, 300), (3001, 17)])
def test_gate_and_column_sums(shape, dtype):
    dq = _dq()
    R, C = shape
    rng = np.random.default_rng(C)
    _said("gate", shape, dtype)
    x, act = _inputs(rng, R, C, hard=False), np.maximum(rng.standard_normal((R, C)), 0)
    if dtype == "f16":
        x = rng.standard_normal((R, C))
    act[:: 5] = 0.0  # rows that nothing comes through
    x = on_gpu(x, TYPES[dtype], C + 1, 1)
    gate = on_gpu(act, TYPES[dtype], C + 2, 1)
    gate[R // 2, 0] = float("nan")  # not above 0
    x[R // 2, 0] = float("nan")
    want = np.where(f64(gate) > 0, f64(x), 0.0)
    q, qt = dq.MxMatrix(R, C, "cuda"), dq.MxMatrix(C, R, "cuda")
    sums = torch.empty(C, device="cuda")
    ws = torch.empty(dq.dqrm_mxfp4_quant_workspace_bytes(R, C), dtype=torch.uint8, device="cuda")
    dq.dqrm_mxfp4_quant(x, q, qt, gate=gate, col_sums=sums, workspace=ws)
    for m, w in ((q, want), (qt, want.T)):
        code, scale = ref.quantise(w)
        c, s = _codes(m)
        np.testing.assert_array_equal(s, scale)
        np.testing.assert_array_equal(c, ref.pack(code))
    # sums of 32 values in turn, four of those, then of every 16th tile of 128 rows, then of 16: no more additions in a chain than
    steps = 32 + 2 + R // (128 * 16) + 1 + 16
    assert np.all(np.abs(f64(sums) - want.sum(0)) <= steps * HALF_ULP["f32"] * 1.01 * np.abs(want).sum(0))
    only = torch.empty(C, device="cuda")
    dq.dqrm_mxfp4_quant(x, gate=gate, col_sums=only, workspace=ws)
    assert torch.equal(only, sums)
    rows_only = dq.MxMatrix(R, C, "cuda")
    dq.dqrm_mxfp4_quant(x, rows_only, gate=gate)
    assert torch.equal(rows_only.codes, q.codes) and torch.equal(rows_only.scales, q.scales)


def test_empty_matrices():
    dq = _dq()
    sums = torch.full((5,), 7.0, device="cuda")
    ws = torch.empty(256, dtype=torch.uint8, device="cuda")
    x = torch.empty((0, 5), device="cuda")
    dq.dqrm_mxfp4_quant(x, dq.MxMatrix(0, 5, "cuda"), dq.MxMatrix(5, 0, "cuda"), col_sums=sums, workspace=ws)
    assert torch.equal(sums, torch.zeros_like(sums))
    dq.dqrm_mxfp4_quant(torch.empty((5, 0), device="cuda"), dq.MxMatrix(5, 0, "cuda"))
    dq.dqrm_mxfp4_dequant(dq.MxMatrix(0, 5, "cuda"), x)
    out, bias = torch.full((3, 4), 7.0, device="cuda"), torch.tensor([1.0, -2.0, float("nan"), 0.5], device="cuda")
    dq.dqrm_mxfp4_matmul(dq.MxMatrix(3, 0, "cuda"), dq.MxMatrix(4, 0, "cuda"), out, bias=bias, relu=True, workspace=ws)
    assert torch.equal(out.nan_to_num(9.0), torch.tensor([[1.0, 0.0, 9.0, 0.5]] * 3, device="cuda"))
    dq.dqrm_mxfp4_matmul(dq.MxMatrix(3, 0, "cuda"), dq.MxMatrix(4, 0, "cuda"), out, workspace=ws)
    assert torch.equal(out, torch.zeros_like(out))
    dq.dqrm_mxfp4_matmul(dq.MxMatrix(0, 64, "cuda"), dq.MxMatrix(4, 64, "cuda"), torch.empty((0, 4), device="cuda"), workspace=ws)
    dq.dqrm_mxfp4_linear(torch.empty((0, 64), device="cuda"), dq.MxMatrix(4, 64, "cuda"), torch.empty((0, 4), device="cuda"), workspace=ws)


# ---- products ---------------------------------------------------------------------------------------------------------


def _held(x):
    dq = _dq()
    code, scale = ref.quantise(x)
    q = dq.MxMatrix(*x.shape, codes=torch.from_numpy(ref.pack(code)).cuda(), scales=torch.from_numpy(scale).cuda())
    return q, ref.values(ref.pack(code), scale, x.shape[1])


def _workspace(n):
    return torch.full((max(int(n), 256),), 0xFF, dtype=torch.uint8, device="cuda")


def _bound(a, b, bias, out, dtype):
    """Sums of 64 products at a time, each of which loses at most two units in the last place of what stands in the sum; partial
    sums of slices of k and the bias in turn; one rounding to the element type."""
    k = a.shape[1]
    size = np.abs(a) @ np.abs(b).T + np.abs(bias)
    return (k / 64 + 40) * 2.0 ** -22 * size + 1.01 * HALF_ULP[dtype] * np.abs(out) + TINY[dtype]


PRODUCTS = [(1, 1, 1), (1, 512, 367), (2, 3, 13), (5, 70, 129), (31, 33, 128), (33, 65, 512), (64, 64, 64), (100, 1, 300), (129, 257, 415),
            (257, 130, 640), (300, 300, 1000), (16, 1000, 2048), (17, 40, 8192), (64, 96, 20000), (512, 367, 8192), (1000, 520, 96), (700, 900, 1537),
            (60, 300, 3000), (50, 5000, 1100), (30, 5000, 200)]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shape", PRODUCTS)
def test_product(shape, dtype):
    dq = _dq()
    m, n, k = shape
    rng = np.random.default_rng(m * 7 + n * 3 + k)
    _said("product", shape, dtype)
    # scales from block to block and row to row, small enough for half precision's outputs
    a, av = _held(rng.standard_normal((m, k)) * np.exp2(rng.integers(-6, 2, (m, 1))) * np.exp2(rng.integers(-3, 1, (1, k))))
    b, bv = _held(rng.standard_normal((n, k)) * np.exp2(rng.integers(-6, 1, (n, 1))))
    bias = rng.standard_normal(n).astype(np.float32)
    ws = _workspace(dq.dqrm_mxfp4_matmul_workspace_bytes(m, n, k))
    for with_bias, relu, stride, offset in ((True, True, n + 3, 1), (False, False, n, 0), (True, False, (n + 7) // 8 * 8, 0)):
        out = on_gpu(np.zeros((m, n)), TYPES[dtype], stride, offset)
        around = out._base.clone()
        dq.dqrm_mxfp4_matmul(a, b, out, bias=torch.from_numpy(bias).cuda() if with_bias else None, relu=relu, workspace=ws)
        add = bias.astype(np.float64) if with_bias else np.zeros(n)
        full = av @ bv.T + add
        want = np.maximum(full, 0) if relu else full
        got = f64(out)
        assert np.all(np.abs(got - want) <= _bound(av, bv, add, want, dtype)), (shape, dtype, np.abs(got - want).max())
        again = torch.empty((m, n), dtype=TYPES[dtype], device="cuda")
        dq.dqrm_mxfp4_matmul(a, b, again, bias=torch.from_numpy(bias).cuda() if with_bias else None, relu=relu, workspace=ws)
        assert torch.equal(again, out)  # the same sums in the same order, whatever the output's stride
        out.fill_(0.0)
        assert torch.equal(out._base.nan_to_num(7.0), around.nan_to_num(7.0))


@pytest.mark.parametrize("shape", [(130, 70, 40000), (70, 600, 33333), (520, 367, 60001), (1030, 770, 40100), (2048, 1000, 60001), (4000, 1000, 65000), (3000, 1100, 700)])
def test_product_of_long_sums_and_of_more_tiles(shape):
    """Slices of k for every side of the tiles, the last one shorter; the plain product in 64 bits on the GPU."""
    dq = _dq()
    m, n, k = shape
    _said("long product", shape)
    gen = torch.Generator("cuda").manual_seed(m + n + k)
    held = []
    for rows in (m, n):
        x = torch.randn((rows, k), device="cuda", generator=gen) * 0.25
        q = dq.MxMatrix(rows, k, "cuda")
        dq.dqrm_mxfp4_quant(x, q)
        dq.dqrm_mxfp4_dequant(q, x)
        held.append((q, x.double()))
    (a, av), (b, bv) = held
    bias = torch.randn(n, device="cuda", generator=gen)
    out = torch.full((m, n), float("nan"), device="cuda")
    dq.dqrm_mxfp4_matmul(a, b, out, bias=bias, relu=True, workspace=_workspace(dq.dqrm_mxfp4_matmul_workspace_bytes(m, n, k)))
    want = (av @ bv.T + bias.double()).clamp_min(0.0)
    size = av.abs() @ bv.abs().T + bias.double().abs()
    bound = (k / 64 + 40) * 2.0 ** -22 * size + 1.01 * HALF_ULP["f32"] * want + TINY["f32"]
    assert bool(((out.double() - want).abs() <= bound).all()), (shape, float((out.double() - want).abs().max()))


@pytest.mark.parametrize("shape", [(3, 70, 300), (200, 150, 600), (40, 30, 9000)])
def test_product_keeps_nans_to_the_rows_that_hold_them(shape):
    dq = _dq()
    m, n, k = shape
    rng = np.random.default_rng(11)
    x, w = rng.standard_normal((m, k)), rng.standard_normal((n, k))
    x[m // 2, k - 1] = np.nan
    x[0, 0] = np.inf
    w[n - 1, k // 2] = -np.inf
    (a, av), (b, bv) = _held(x), _held(w)
    for relu in (False, True):
        out = torch.empty((m, n), device="cuda")
        dq.dqrm_mxfp4_matmul(a, b, out, relu=relu, workspace=_workspace(dq.dqrm_mxfp4_matmul_workspace_bytes(m, n, k)))
        want = np.isnan(av).any(1)[:, None] | np.isnan(bv).any(1)[None, :]
        np.testing.assert_array_equal(np.isnan(f64(out)), want)


def test_product_of_operands_that_are_all_zero():
    dq = _dq()
    a, _ = _held(np.zeros((40, 200)))
    b, _ = _held(np.random.default_rng(0).standard_normal((70, 200)))
    out = torch.full((40, 70), 5.0, device="cuda")
    dq.dqrm_mxfp4_matmul(a, b, out, workspace=_workspace(dq.dqrm_mxfp4_matmul_workspace_bytes(40, 70, 200)))
    assert torch.equal(out, torch.zeros_like(out))


# ---- a linear layer on activations ----------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shape", [(1, 1, 1), (1, 512, 367), (1, 300, 8192), (2, 70, 13), (4, 1000, 1000), (7, 33, 129), (16, 512, 2048), (17, 100, 64),
                                   (33, 300, 300), (64, 65, 4097), (200, 130, 415), (1, 40, 20000)])
def test_linear_is_quantisation_and_product(shape, dtype):
    dq = _dq()
    m, n, k = shape
    rng = np.random.default_rng(m + n + k)
    _said("linear", shape, dtype)
    w, wv = _held(rng.standard_normal((n, k)) / np.sqrt(k))
    bias = rng.standard_normal(n).astype(np.float32)
    ws = _workspace(dq.dqrm_mxfp4_linear_workspace_bytes(m, n, k))
    for stride, offset, relu in ((k, 0, True), (k + 5, 3, False)):
        x = on_gpu(rng.standard_normal((m, k)) * np.exp2(rng.integers(-4, 2, (m, 1))), TYPES[dtype], stride, offset)
        out = on_gpu(np.zeros((m, n)), TYPES[dtype], n + 3, 1)
        around = out._base.clone()
        dq.dqrm_mxfp4_linear(x, w, out, bias=torch.from_numpy(bias).cuda(), relu=relu, workspace=ws)
        xv = ref.quantised_values(f64(x))
        want = xv @ wv.T + bias
        want = np.maximum(want, 0) if relu else want
        assert np.all(np.abs(f64(out) - want) <= _bound(xv, wv, bias, want, dtype))
        out.fill_(0.0)
        assert torch.equal(out._base.nan_to_num(7.0), around.nan_to_num(7.0))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shape", [(1, 1, 2), (1, 200, 367), (3, 64, 8192), (16, 300, 1000), (40, 33, 515), (1, 16, 40000)])
def test_linear_behind_a_norm(shape, dtype):
    """The norm's sums may differ from the reference's in their last bits, and a value that lies that near to a boundary between
    two codes takes either: rows whose values keep their distance from boundaries are held to the product's bound, the others to
    a step between codes at each value that does not."""
    dq = _dq()
    m, n, k = shape
    rng = np.random.default_rng(k)
    _said("norm + linear", shape, dtype)
    w, wv = _held(rng.standard_normal((n, k)) / np.sqrt(k))
    x = on_gpu(rng.standard_normal((m, k)) * 3 + 1, TYPES[dtype], k + 1, 1)
    gamma, beta = (1 + 0.3 * rng.standard_normal(k)).astype(np.float32), rng.standard_normal(k).astype(np.float32)
    for g, b in ((gamma, beta), (None, None)):
        y, mean, rstd = ref.norm(f64(x), 1.0 if g is None else g.astype(np.float64), 0.0 if b is None else b.astype(np.float64), 1e-5)
        out = torch.empty((m, n), dtype=TYPES[dtype], device="cuda")
        put = lambda v: None if v is None else torch.from_numpy(v).cuda()  # noqa: E731
        dq.dqrm_mxfp4_linear(x, w, out, gamma=put(g), beta=put(b), eps=1e-5, workspace=_workspace(dq.dqrm_mxfp4_linear_workspace_bytes(m, n, k)))
        # how far a 32-bit y may be off (see the norm's own test), and which codes that lets through
        off = 2.0 ** -18 * (np.abs(y) + np.abs(f64(x)).max(1, keepdims=True) * rstd[:, None] * (1.0 if g is None else np.abs(g)) + (0.0 if b is None else np.abs(b)))
        yv = ref.quantised_values(y)
        spread = np.abs(ref.quantised_values(y + off) - yv) + np.abs(ref.quantised_values(y - off) - yv)
        # (a block's scale changes if its maximum crosses a power of two: then every value of it may take another code)
        top = np.zeros((m, ref.pad128(k)))
        top[:, :k] = np.abs(y)
        amax = top.reshape(m, -1, 32).max(-1)
        room = np.zeros((m, ref.pad128(k)))
        room[:, :k] = off
        near = np.abs(amax - np.exp2(np.round(np.log2(np.maximum(amax, 1e-30))))) <= room.reshape(m, -1, 32).max(-1)
        wide = np.repeat(near, 32, 1)[:, :k] * np.repeat(amax, 32, 1)[:, :k]
        want = yv @ wv.T
        may = _bound(yv, wv, np.zeros(n), want, dtype) + (spread + wide) @ np.abs(wv).T * (1 + HALF_ULP[dtype])
        assert np.all(np.abs(f64(out) - want) <= may)


def test_gradients_of_a_layer_against_differences():
    """Loss = sum of dz (X W^T + b) with operands that the format holds: its differences are the products' gradients."""
    dq = _dq()
    rng = np.random.default_rng(8)
    M, N, K = 160, 96, 130
    draw = lambda r, c: rng.choice(ref.MAGNITUDES, (r, c)) * rng.choice([-1.0, 1.0], (r, c))  # noqa: E731
    X, W, dz = draw(M, K), draw(N, K), draw(M, N)
    for a in (X, W, dz):  # every block, in both directions, has a 4 or a 6: its scale is 1 and it is held exactly
        a[::7, :], a[:, ::7] = 4.0, 6.0
    put = lambda a: torch.from_numpy(a).float().cuda()  # noqa: E731
    x_t, w_t = dq.MxMatrix(K, M, "cuda"), dq.MxMatrix(K, N, "cuda")
    dq.dqrm_mxfp4_quant(put(X), None, x_t)
    dq.dqrm_mxfp4_quant(put(W), None, w_t)
    q, q_t, db = dq.MxMatrix(M, N, "cuda"), dq.MxMatrix(N, M, "cuda"), torch.empty(N, device="cuda")
    ws = _workspace(max(dq.dqrm_mxfp4_quant_workspace_bytes(M, N), dq.dqrm_mxfp4_matmul_workspace_bytes(M, K, N), dq.dqrm_mxfp4_matmul_workspace_bytes(N, K, M)))
    dq.dqrm_mxfp4_quant(put(dz), q, q_t, col_sums=db, workspace=ws)
    dx, dw = torch.empty((M, K), device="cuda"), torch.empty((N, K), device="cuda")
    dq.dqrm_mxfp4_matmul(q, w_t, dx, workspace=ws)
    dq.dqrm_mxfp4_matmul(q_t, x_t, dw, workspace=ws)
    b = np.zeros(N)
    loss = lambda X, W, b: float((dz * (X @ W.T + b)).sum())  # noqa: E731
    for arr, grad in ((X, f64(dx)), (W, f64(dw)), (b, f64(db))):
        for _ in range(25):
            at = tuple(int(rng.integers(0, s)) for s in arr.shape)
            old = arr[at]
            arr[at] = old + 0.5
            up = loss(X, W, b)
            arr[at] = old - 0.5
            down = loss(X, W, b)
            arr[at] = old
            assert up - down == grad[at]  # linear in each, and all of it is exact


# ---- streams, graphs, sizes past 32 bits ------------------------------------------------------------------------------------


def test_on_another_stream_and_in_a_graph():
    dq = _dq()
    rng = np.random.default_rng(2)
    M, N, K = 300, 200, 5000
    x = torch.from_numpy(rng.standard_normal((M, K))).float().cuda()
    w = torch.from_numpy(rng.standard_normal((N, K))).float().cuda()
    gamma = torch.ones(K, device="cuda")
    qx, qw, qt = dq.MxMatrix(M, K, "cuda"), dq.MxMatrix(N, K, "cuda"), dq.MxMatrix(K, M, "cuda")
    out, few, sums = torch.empty((M, N), device="cuda"), torch.empty((4, N), device="cuda"), torch.empty(K, device="cuda")
    dx, dg, db = torch.empty_like(x), torch.empty(K, device="cuda"), torch.empty(K, device="cuda")
    mean, rstd = torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    ws = _workspace(max(dq.dqrm_mxfp4_quant_workspace_bytes(M, K), dq.dqrm_mxfp4_matmul_workspace_bytes(M, N, K),
                        dq.dqrm_mxfp4_linear_workspace_bytes(4, N, K), dq.dqrm_layernorm_bwd_workspace_bytes(M, K)))

    def work():
        dq.dqrm_mxfp4_quant(w, qw)
        dq.dqrm_layernorm_fwd(x, gamma, None, 1e-5, mean=mean, rstd=rstd, q=qx)
        dq.dqrm_mxfp4_quant(x, None, qt, col_sums=sums, workspace=ws)
        dq.dqrm_mxfp4_matmul(qx, qw, out, workspace=ws)
        dq.dqrm_mxfp4_linear(x[:4], qw, few, gamma=gamma, eps=1e-5, workspace=ws)
        dq.dqrm_layernorm_bwd(x, x, mean, rstd, gamma, dx, dg, db, ws)

    results = (qx.codes, qx.scales, qw.codes, qt.codes, out, few, sums, dx, dg, db, mean, rstd)
    work()
    torch.cuda.synchronize()
    want = [t.clone() for t in results]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for t in results:
            t.zero_()
        work()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(results, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for k in range(4):
        for t in results:
            t.zero_()
        x.mul_(2.0 if k % 2 else 1.0)  # work between the replays
        x.div_(2.0 if k % 2 else 1.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(results, want)), k


@pytest.mark.parametrize("cols", [1, 3, 7, 65])
def test_operands_that_end_where_their_memory_ends(cols):
    """Allocations of whole mebibytes that a matrix fills to the last byte: vectors of rows shorter than a vector, half stages of k and
    rows past the last one must not be asked for."""
    dq = _dq()
    rng = np.random.default_rng(cols)
    R = (20 << 20) // 2 // cols // 64 * 64
    x = torch.empty(R * cols, dtype=torch.bfloat16, device="cuda").view(R, cols)
    x.normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    few = [0, 1, R // 2, R - 9, R - 2, R - 1]
    _said("quantise", R, cols)
    q, qt = dq.MxMatrix(R, cols, "cuda"), dq.MxMatrix(cols, R, "cuda")
    sums, ws = torch.empty(cols, device="cuda"), _workspace(dq.dqrm_mxfp4_quant_workspace_bytes(R, cols))
    dq.dqrm_mxfp4_quant(x, q)
    dq.dqrm_mxfp4_quant(x, None, qt, gate=x, col_sums=sums, workspace=ws)
    code, scale = ref.quantise(f64(x[few]))
    np.testing.assert_array_equal(q.scales[few].cpu().numpy(), scale)
    np.testing.assert_array_equal(q.codes[few].cpu().numpy(), ref.pack(code))
    code, scale = ref.quantise(np.maximum(f64(x), 0).T)
    np.testing.assert_array_equal(qt.scales.cpu().numpy(), scale)
    np.testing.assert_array_equal(qt.codes.cpu().numpy(), ref.pack(code))
    # W of 20 MiB of codes (one group of 128 values to a row), as the second operand of a large and of a small product
    N = (20 << 20) // 64
    w = dq.MxMatrix(N, cols, "cuda")
    wv = rng.choice(ref.MAGNITUDES, (N, cols)) * rng.choice([-1.0, 1.0], (N, cols))
    dq.dqrm_mxfp4_quant(torch.from_numpy(wv).to(torch.bfloat16).cuda(), w)
    wv = ref.quantised_values(wv)
    for m in (70, 3):
        a, av = _held(rng.standard_normal((m, cols)))
        out = torch.empty((m, N), dtype=torch.bfloat16, device="cuda")
        _said("product", m, N, cols)
        dq.dqrm_mxfp4_matmul(a, w, out, workspace=_workspace(dq.dqrm_mxfp4_matmul_workspace_bytes(m, N, cols)))
        want = av @ wv.T
        assert np.all(np.abs(f64(out) - want) <= _bound(av, wv, np.zeros(N), want, "bf16"))
        out = torch.empty((N, m), dtype=torch.bfloat16, device="cuda")
        _said("product", N, m, cols)
        dq.dqrm_mxfp4_matmul(w, a, out, workspace=_workspace(dq.dqrm_mxfp4_matmul_workspace_bytes(N, m, cols)))
        assert np.all(np.abs(f64(out) - want.T) <= _bound(wv, av, np.zeros(m), want.T, "bf16"))


def test_offsets_past_32_bits():
    dq = _dq()
    R, C = 70001, 65600  # 4.6 G values
    x = torch.empty((R, C), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    few = [0, 1, 32767, 32768, 65535, 65536, R - 2, R - 1]
    for r0 in range(0, R, 8192):
        x[r0:r0 + 8192].normal_(generator=g)
    q, qt = dq.MxMatrix(R, C, "cuda"), dq.MxMatrix(C, R, "cuda")
    sums = torch.empty(C, device="cuda")
    ws = _workspace(dq.dqrm_mxfp4_quant_workspace_bytes(R, C))
    _said("quantise", R, C)
    dq.dqrm_mxfp4_quant(x, q, qt, col_sums=sums, workspace=ws)
    code, scale = ref.quantise(f64(x[few]))
    np.testing.assert_array_equal(q.scales[few].cpu().numpy(), scale)
    np.testing.assert_array_equal(q.codes[few].cpu().numpy(), ref.pack(code))
    cols = [0, 65535, 65536, C - 1]
    sub = f64(x[:, cols]).T
    code, scale = ref.quantise(sub)
    np.testing.assert_array_equal(qt.scales[cols].cpu().numpy(), scale)
    np.testing.assert_array_equal(qt.codes[cols].cpu().numpy(), ref.pack(code))
    assert np.all(np.abs(f64(sums[cols]) - sub.sum(1)) <= (32 + 2 + R // 2048 + 17) * HALF_ULP["f32"] * 1.01 * np.abs(sub).sum(1))
    rows_only = dq.MxMatrix(R, C, "cuda")
    dq.dqrm_mxfp4_quant(x, rows_only)
    assert torch.equal(rows_only.codes, q.codes) and torch.equal(rows_only.scales, q.scales)
    del rows_only, qt
    y = torch.empty_like(x)
    _said("dequantise")
    dq.dqrm_mxfp4_dequant(q, y)
    np.testing.assert_array_equal(f64(y[few]), ref.quantised_values(f64(x[few])))
    # a product whose first operand's codes and whose outputs pass 2^31 and 2^32 bytes
    w, wv = _held(np.random.default_rng(5).standard_normal((257, C)) / np.sqrt(C))
    out = torch.empty((R, 40000), dtype=torch.bfloat16, device="cuda")[:, :257]
    ws = _workspace(dq.dqrm_mxfp4_matmul_workspace_bytes(R, 257, C))
    _said("product")
    dq.dqrm_mxfp4_matmul(q, w, out, workspace=ws)
    av = ref.quantised_values(f64(x[few]))
    want = av @ wv.T
    assert np.all(np.abs(f64(out[few]) - want) <= _bound(av, wv, np.zeros(257), want, "bf16"))
    mean, rstd = torch.empty(R, device="cuda"), torch.empty(R, device="cuda")
    _said("norm")
    dq.dqrm_layernorm_fwd(x, None, None, 1e-5, y=y, mean=mean, rstd=rstd)
    yv, mv, rv = ref.norm(f64(x[few]), 1.0, 0.0, 1e-5)
    assert np.all(np.abs(f64(y[few]) - yv) <= 2.0 ** -8 * np.abs(yv) + 1e-5)
    dgamma, dbeta = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    ws = _workspace(dq.dqrm_layernorm_bwd_workspace_bytes(R, C))
    dq.dqrm_layernorm_bwd(x, x, mean, rstd, None, y, dgamma, dbeta, ws)
    dxv, _, _ = ref.norm_backward(f64(x[few]), f64(x[few]), f64(mean[few]), f64(rstd[few]), 1.0)
    assert np.all(np.abs(f64(y[few]) - dxv) <= backward_bounds(f64(x[few]), f64(x[few]), f64(mean[few]), f64(rstd[few]), 1.0, dxv, "bf16", 1)[0])
    chain = -(-R // 64) + 64
    assert np.all(np.abs(f64(dbeta[cols]) - sub.sum(1)) <= chain * HALF_ULP["f32"] * np.abs(sub).sum(1))
