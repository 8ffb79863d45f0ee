"""Softmax cross entropy over many classes against its definition in 64 bits."""
import math

import pytest
import torch

import paper_2410_20046_amd as dq
from xent_reference import gradients_and_bounds, loss_and_bounds, near

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def space(n):
    return torch.empty(max(n, 1), dtype=torch.uint8, device="cuda").fill_(0xFF)  # (NaNs, wherever something is read that nobody wrote)


BEHIND = 4096


def untouched(room):
    assert bool((room[-BEHIND:] == 0xFF).all()), "written behind the workspace"


def forward(x, w, targets, bias=None, scale=1.0, stream=None):
    m, v, k = x.shape[0], w.shape[0], x.shape[1]
    loss, lse = (torch.full((m,), math.nan, device="cuda") for _ in range(2))
    room = space(dq.dqrm_softmax_xent_fwd_workspace_bytes(m, v, k, x.dtype) + BEHIND)
    dq.dqrm_softmax_xent_fwd(x, w, targets, loss, lse, bias=bias, scale=scale, workspace=room[:-BEHIND], stream=stream)
    untouched(room)
    return loss, lse


def backward(x, w, targets, lse, grad, bias=None, scale=1.0):
    m, v, k = x.shape[0], w.shape[0], x.shape[1]
    dx, dw = torch.full_like(x, math.nan).contiguous(), torch.full((v, k), math.nan, dtype=x.dtype, device="cuda")
    dbias = torch.full((v,), math.nan, device="cuda")
    room = space(dq.dqrm_softmax_xent_bwd_workspace_bytes(m, v, k, x.dtype) + BEHIND)
    dq.dqrm_softmax_xent_bwd(x, w, targets, lse, grad, dx=dx, dw=dw, dbias=dbias, bias=bias, scale=scale, workspace=room[:-BEHIND])
    untouched(room)
    return dx, dw, dbias


def make(m, v, k, dtype, seed=0, bias=True, spread=1.5):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn(m, k, device="cuda", generator=g).to(dtype)
    w = (torch.randn(v, k, device="cuda", generator=g) * spread / math.sqrt(max(k, 1))).to(dtype)
    targets = torch.randint(0, v, (m,), device="cuda", generator=g)
    b = torch.randn(v, device="cuda", generator=g) if bias else None
    grad = torch.rand(m, device="cuda", generator=g) / m
    return x, w, targets, b, grad


def check(x, w, targets, bias, scale, grad):
    loss, lse = forward(x, w, targets, bias, scale)
    r = gradients_and_bounds(x, w, targets, bias, scale, grad)
    near(lse, r["lse"], r["lse_off"], "lse")
    near(loss, r["loss"], r["loss_off"], "loss")
    dx, dw, dbias = backward(x, w, targets, lse, grad, bias, scale)
    near(dbias, *r["dbias"], "dbias")
    near(dx, *r["dx"], "dx")
    near(dw, *r["dw"], "dw")


# rows, classes, width: single ones, parts of tiles, several tiles, each shape of tile, sums in slices, several pieces of the classes
SHAPES = [(1, 1, 1), (1, 1000, 16), (3, 7, 5), (17, 257, 64), (64, 300, 200), (65, 300, 64), (130, 513, 72), (300, 1000, 40), (257, 700, 1021), (2, 35, 1059),
          (64, 20000, 40), (1000, 12, 22), (5000, 40, 300), (600, 33000, 96), (129, 100, 2048), (520, 33000, 600), (8300, 700, 1100), (40, 100, 100),
          (30, 50, 100), (20, 200, 50), (17000, 40, 24), (100, 200, 100), (100, 500, 100), (300, 5000, 200), (5000, 300, 200),
          (30, 200, 96), (40, 300, 61), (33, 9000, 130), (64, 70001, 41), (7, 4500, 1021), (30, 200, 40),
          (100, 300, 16), (200, 5000, 32), (70, 500, 9), (65, 64, 33), (1025, 129, 1), (128, 20000, 64), (129, 130, 48),
          (233, 27, 5541), (8, 1118, 6953), (64, 5, 2080), (65, 1000, 4096), (1000, 700, 2056), (1, 1, 9000), (40, 3000, 2100)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m, v, k", SHAPES)
def test_loss_and_gradients(m, v, k, dtype):
    x, w, targets, bias, grad = make(m, v, k, TYPES[dtype], seed=m + v + k)
    check(x, w, targets, bias, 0.75, grad)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m", [1, 2, 3, 4, 5, 8, 9, 16])
def test_a_few_rows(m, dtype):
    """Each number of rows of the kernel for a few of them, several times that many, one lane to a class and a whole wave, and more classes than
    its workgroups take at once."""
    for v, k in ((5, 8), (3000, 3), (3001, 61), (9, 515), (70001, 17), (40, 9001)):
        x, w, targets, bias, grad = make(m, v, k, TYPES[dtype], seed=m + v)
        bias[v // 2] = -math.inf
        targets[0] = -1
        loss, lse = forward(x, w, targets, bias, 1.25)
        r = loss_and_bounds(x, w, targets, bias, 1.25)
        near(lse, r["lse"], r["lse_off"], "lse")
        near(loss, r["loss"], r["loss_off"], "loss")


# more classes than a piece takes, of d or of rows of w that have to be laid out anew
PIECES = [(t, 8001, 40000, k) for t in ("bf16", "f16") for k in (32, 72, 160)] + [("f32", 3001, 40000, 24), ("bf16", 30, 70000, 4104), ("f16", 30, 70000, 4104),
                                                                                                  ("f32", 30, 30000, 4104), ("f32", 50, 30000, 4104), ("f32", 70, 1500000, 8)]


@pytest.mark.parametrize("dtype, m, v, k", PIECES)
def test_classes_in_several_pieces(dtype, m, v, k):
    """d, or the rows of w that have to be laid out anew, take more than a piece's room."""
    x, w, targets, _, grad = make(m, v, k, TYPES[dtype], seed=3, bias=False)
    check(x, w, targets, None, 1.0, grad)


@pytest.mark.parametrize("dtype", TYPES)
def test_strides_and_alignment(dtype):
    """Rows with gaps, and matrices that begin anywhere, give what contiguous ones give, and nothing is written beside the outputs."""
    m, v, k = 70, 530, 88
    t = TYPES[dtype]
    x, w, targets, bias, grad = make(m, v, k, t, seed=9)
    loss, lse = forward(x, w, targets, bias)
    dx, dw, dbias = backward(x, w, targets, lse, grad, bias)
    for shift, gap in ((0, 8), (0, 3), (1, 7), (5, 11)):
        def put(a):
            big = torch.full((a.shape[0] + 1, k + gap), math.nan, dtype=t, device="cuda")
            view = big.view(-1)[shift:shift + a.shape[0] * (k + gap)].view(a.shape[0], k + gap)[:, :k]
            view.copy_(a)
            return big, view
        (_, xs), (_, ws) = put(x), put(w)
        loss2, lse2 = forward(xs, ws, targets, bias)
        assert torch.equal(loss, loss2) and torch.equal(lse, lse2)
        (bx, dxs), (bw, dws) = put(torch.zeros_like(x)), put(torch.zeros_like(w))
        before = torch.isnan(bx).sum(), torch.isnan(bw).sum()
        db = torch.empty_like(dbias)
        dq.dqrm_softmax_xent_bwd(xs, ws, targets, lse, grad, dx=dxs, dw=dws, dbias=db, bias=bias,
                                 workspace=space(dq.dqrm_softmax_xent_bwd_workspace_bytes(m, v, k, t)))
        assert torch.equal(dxs, dx) and torch.equal(dws, dw) and torch.equal(db, dbias)
        assert (torch.isnan(bx).sum(), torch.isnan(bw).sum()) == before


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m, v, k", [(70, 900, 48), (3, 130, 17), (70, 900, 120), (40, 900, 75), (200, 600, 200), (30, 500, 40), (70, 900, 2052), (20, 500, 2056)])
def test_rows_without_target_and_classes_taken_out(m, v, k, dtype):
    """Rows without a target, with a gradient of zero, classes with a bias of -infinity: whatever x and w hold there."""
    t = TYPES[dtype]
    x, w, targets, bias, grad = make(m, v, k, t, seed=5)
    out = torch.arange(v, device="cuda") % 7 == 3
    bias[out] = -math.inf
    targets[targets % 7 == 3] -= 1
    targets[1], targets[2] = -1, -(1 << 40)
    grad[0] = 0
    for inside in (False, True):
        if inside:  # garbage where nothing counts
            w[out] = math.nan
            w[3, 0] = math.inf
            x[1], x[2] = math.nan, math.inf
        clean_w, clean_x = torch.where(out[:, None], torch.zeros_like(w), w), x.clone()
        clean_x[1:3] = 0
        loss, lse = forward(x, w, targets, bias)
        r = gradients_and_bounds(clean_x, clean_w, targets, bias, 1.0, grad)
        near(loss, r["loss"], r["loss_off"], "loss")
        assert bool((loss[1:3] == 0).all())
        keep = torch.ones(m, dtype=torch.bool, device="cuda")
        keep[1:3] = False
        near(lse[keep], r["lse"][keep], r["lse_off"][keep], "lse")
        dx, dw, dbias = backward(x, w, targets, lse, grad, bias)
        near(dx, *r["dx"], "dx")
        near(dw, *r["dw"], "dw")
        near(dbias, *r["dbias"], "dbias")
        assert bool((dx[:3] == 0).all()) and bool((dbias[out] == 0).all()) and bool((dw[out] == 0).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m, k", [(5, 24), (100, 24), (100, 136), (40, 75), (100, 2052)])
def test_rows_with_no_class_left(m, k, dtype):
    x, w, targets, _, grad = make(m, 300, k, TYPES[dtype], seed=6)
    bias = torch.full((300,), -math.inf, device="cuda")
    loss, lse = forward(x, w, targets, bias)
    assert bool((lse == -math.inf).all()) and bool((loss == math.inf).all())
    for out in backward(x, w, targets, lse, grad, bias):
        assert bool((out == 0).all())
    # the targets alone are taken out
    bias = torch.zeros(300, device="cuda")
    bias[targets] = -math.inf
    r = gradients_and_bounds(x, w, targets, bias, 1.0, grad)
    loss, lse = forward(x, w, targets, bias)
    assert bool((loss == math.inf).all())
    near(lse, r["lse"], r["lse_off"], "lse")
    dx, _, dbias = backward(x, w, targets, lse, grad, bias)
    near(dbias, *r["dbias"], "dbias")
    near(dx, *r["dx"], "dx")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m, k", [(140, 24), (140, 136), (60, 75), (60, 24), (140, 2052)])
def test_infinities_and_nans_stay_in_their_rows(m, k, dtype):
    x, w, targets, bias, grad = make(m, 300, k, TYPES[dtype], seed=7)
    loss0, _ = forward(x, w, targets, bias)
    x[m // 2 + 7, 3] = math.nan
    x[12, 5] = math.inf
    loss, lse = forward(x, w, targets, bias)
    bad = torch.zeros(m, dtype=torch.bool, device="cuda")
    bad[[12, m // 2 + 7]] = True
    assert bool(torch.isnan(loss[bad]).all()) and bool(torch.isnan(lse[bad]).all()) and torch.equal(loss[~bad], loss0[~bad])
    dx, dw, dbias = backward(x, w, targets, lse, grad, bias)
    assert bool(torch.isnan(dx[bad]).all()) and not bool(torch.isnan(dx[~bad]).any()) and bool(torch.isnan(dbias).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m, k", [(33, 64), (133, 64), (133, 200)])
def test_large_logits(m, k, dtype):
    """Far beyond where exponentials overflow; a row whose one class has all the weight; a loss near zero."""
    x, w, targets, bias, grad = make(m, 400, k, TYPES[dtype], seed=8, spread=300.0)
    check(x, w, targets, bias, 1.0, grad)
    l = x.double() @ w.double().t() + bias.double()
    check(x, w, l.argmax(1), bias, 1.0, grad)


@pytest.mark.parametrize("k", [40, 104])
def test_gradients_of_very_different_sizes_in_half(k):
    """fp16 keeps d times a power of two: the smallest rows' gradients are there, down to 2^-40 of the largest."""
    x, w, targets, bias, _ = make(200, 300, k, torch.float16, seed=10)
    grad = torch.exp2(-torch.arange(200, device="cuda").float() / 12) * 1e-5
    check(x, w, targets, bias, 1.0, grad)
    grad = torch.full((200,), 2.0 ** -130, device="cuda")
    check(x, w, targets, bias, 1.0, grad)
    grad = torch.full((200,), 100.0, device="cuda")
    check(x, w, targets, bias, 1.0, grad)


@pytest.mark.parametrize("m, k", [(40, 24), (40, 75), (140, 24), (140, 136)])
def test_a_target_past_the_last_class_is_recorded(m, k):
    x, w, targets, bias, grad = make(m, 300, k, torch.bfloat16, seed=11)
    dq.dqrm_check_status()
    good = targets.clone()
    good[17] = -1
    loss0, lse0 = forward(x, w, good, bias)
    assert dq.dqrm_check_status()[0] == 0
    targets[17] = 300
    loss, lse = forward(x, w, targets, bias)
    assert dq.dqrm_check_status() == (dq.ERR_INDEX_OUT_OF_RANGE, -1, 300) and dq.dqrm_check_status()[0] == 0
    assert torch.equal(loss, loss0) and torch.equal(lse, lse0)
    for a, b in zip(backward(x, w, targets, lse, grad, bias), backward(x, w, good, lse, grad, bias)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("k", [24, 136])
def test_outputs_one_by_one_and_empty_calls(k, dtype):
    t = TYPES[dtype]
    x, w, targets, bias, grad = make(70, 300, k, t, seed=12)
    _, lse = forward(x, w, targets, bias)
    dx, dw, dbias = backward(x, w, targets, lse, grad, bias)
    ws = space(dq.dqrm_softmax_xent_bwd_workspace_bytes(70, 300, k, t))
    for name, want in (("dx", dx), ("dw", dw), ("dbias", dbias)):
        got = torch.full_like(want, math.nan)
        dq.dqrm_softmax_xent_bwd(x, w, targets, lse, grad, bias=bias, workspace=ws, **{name: got})
        assert torch.equal(got, want), name
    # no rows: gradients of zeros
    none = x[:0], w, targets[:0]
    forward(*none, bias)
    ex, ew, eb = backward(*none, lse[:0], grad[:0], bias)
    assert ex.shape == (0, k) and bool((ew == 0).all()) and bool((eb == 0).all())
    # no width: the bias alone
    loss, lse = forward(x[:, :0], w[:, :0], targets, bias)
    want = torch.logsumexp(bias.double(), 0)
    near(lse, want.expand(70), torch.full((70,), 2.0 ** -24 * 300, device="cuda"), "lse")
    near(loss, want - bias.double()[targets], torch.full((70,), 2.0 ** -24 * 300, device="cuda"), "loss")


@pytest.mark.parametrize("m, v, k", [(300, 5000, 64), (300, 5000, 136), (20, 5000, 75), (30, 300, 2056)])
def test_equal_on_another_stream_and_replayed(m, v, k):
    x, w, targets, bias, grad = make(m, v, k, torch.bfloat16, seed=13)
    loss, lse = forward(x, w, targets, bias)
    want = [loss, lse, *backward(x, w, targets, lse, grad, bias)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        loss2, lse2 = forward(x, w, targets, bias)
        got = [loss2, lse2, *backward(x, w, targets, lse2, grad, bias)]
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    out = [torch.empty_like(t) for t in want]
    ws = [space(f(m, v, k, x.dtype)) for f in (dq.dqrm_softmax_xent_fwd_workspace_bytes, dq.dqrm_softmax_xent_bwd_workspace_bytes)]

    def step():
        dq.dqrm_softmax_xent_fwd(x, w, targets, out[0], out[1], bias=bias, workspace=ws[0])
        dq.dqrm_softmax_xent_bwd(x, w, targets, out[1], grad, dx=out[2], dw=out[3], dbias=out[4], bias=bias, workspace=ws[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(4):
        x.copy_(torch.randn_like(x))
        targets.copy_(torch.randint_like(targets, -2, v))
        for t in out:
            t.fill_(math.nan)
        graph.replay()
        torch.cuda.synchronize()
        loss, lse = forward(x, w, targets, bias)
        want = [loss, lse, *backward(x, w, targets, lse, grad, bias)]
        assert all(torch.equal(a, b) for a, b in zip(want, out)), turn


def test_gradients_against_differences():
    x, w, targets, bias, _ = make(6, 50, 9, torch.float32, seed=14)
    grad = torch.rand(6, device="cuda") + 0.5
    _, lse = forward(x, w, targets, bias, 0.5)
    dx, dw, dbias = backward(x, w, targets, lse, grad, bias, 0.5)
    f = lambda a, b, c: float((loss_and_bounds(a, b, targets, c, 0.5)["loss"] * grad.double()).sum())  # noqa: E731
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    for of, got in ((0, dx), (1, dw), (2, dbias)):
        args = [x.double(), w.double(), bias.double()]
        way = torch.randn(args[of].shape, device="cuda", dtype=torch.float64, generator=g)
        h = 1e-5
        up, down = list(args), list(args)
        up[of], down[of] = args[of] + h * way, args[of] - h * way
        slope = (f(*up) - f(*down)) / (2 * h)
        # third derivatives of the loss are below 1, h^2 1e-10, and the gradients' own bounds are far below 1e-5
        assert abs(slope - float((got.double() * way).sum())) <= 1e-5 * float((got.double().abs() * way.abs()).sum() + 1)
