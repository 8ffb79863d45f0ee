"""Residual joins with their norms, forward and backward, against their formulas in 64 bits."""
import math

import pytest
import torch

import paper_2410_20046_amd as dq
import resnorm_reference as ref
from mx_reference import TYPES
from xent_reference import near

pytestmark = pytest.mark.gpu
KINDS = {"none": dq.NORM_NONE, "layer": dq.NORM_LAYER, "rms": dq.NORM_RMS}
EPS = 1e-5
# every way a row is laid over threads, both sides of each limit, and more rows than workgroups
SHAPES = [(1, 1), (5, 2), (130, 7), (3, 8), (37, 9), (600, 128), (16, 129), (33, 512), (9, 513), (6, 1024), (7, 1025), (700, 2048), (5, 2049), (300, 4096), (3, 4097),
          (530, 8191), (2, 8192), (3, 8193), (280, 16384)]
MANY = [(4100, 100), (4097, 500), (4100, 1024), (4096, 2000), (4099, 4096), (4100, 8001), (4096, 9000)]
BOTH = [("none", "layer"), ("none", "rms"), ("layer", "none"), ("rms", "none"), ("layer", "layer"), ("rms", "rms"), ("layer", "rms"), ("rms", "layer"), ("none", "none")]


def matrix(a, gap=0, shift=0):
    """`a` in memory of its own with a row stride and a first element, NaN around it"""
    R, C = a.shape
    room = torch.full((shift + R * (C + gap) + 16,), math.nan, dtype=a.dtype, device="cuda")
    view = room[shift:shift + R * (C + gap)].view(R, C + gap)[:, :C]
    view.copy_(a)
    return view


def make(R, C, dtype, post, pre, vectors, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rand = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    t = TYPES[dtype]
    u, r = (rand(R, C) * torch.exp2(rand(R, 1)) + 0.5).to(t), (rand(R, C) * 2).to(t)
    dout, dy = rand(R, C).to(t), (rand(R, C) * torch.exp2(rand(R, 1))).to(t)
    v = dict(post_gamma=1 + 0.3 * rand(C), post_beta=0.2 * rand(C), gate=0.5 + rand(C), pre_gamma=1 + 0.3 * rand(C), pre_beta=0.2 * rand(C))
    if not vectors:
        v = dict.fromkeys(v)
    for side, kind in (("post", post), ("pre", pre)):
        if kind == "none":
            v[side + "_gamma"] = v[side + "_beta"] = None
    p = dict(post=post, pre=pre, res_scale=0.75, eps=EPS)
    for name, value in v.items():
        p[name] = value.double() if value is not None else torch.full((C,), 0.0 if "beta" in name else 1.0, dtype=torch.float64, device="cuda")
    block = dq.ResidualNorm(post=KINDS[post], pre=KINDS[pre], res_scale=0.75, post_eps=EPS, pre_eps=EPS, **v)
    return block, p, u, r, dout, dy


def space(R, C):
    return torch.full((max(dq.dqrm_residual_norm_bwd_workspace_bytes(R, C), 1),), 0xFF, dtype=torch.uint8, device="cuda")


def check_forward(block, p, u, r, out, y, stats):
    dtype = u.dtype
    want = ref.forward(p, u.double(), r.double())
    near(out, want["out"][0], ref.rounded(*want["out"], dtype), "out")
    if p["pre"] != "none":
        near(y, want["y"][0], ref.rounded(*want["y"], dtype), "y")
    for k, (value, off) in enumerate(want["stats"]):
        if value is None:
            assert bool(torch.isnan(stats[k]).all())  # as it was
        else:
            near(stats[k], value[:, 0], 2 * off[:, 0] + 1e-37, f"statistic {k}")


def check_backward(p, dout, dy, u, out, stats, du, dr, dparams):
    want = ref.backward(p, dout.double(), dy.double(), u.double(), out.double(), stats.double())
    near(du, want["du"][0], ref.rounded(*want["du"], u.dtype), "du")
    near(dr, want["dr"][0], ref.rounded(*want["dr"], u.dtype), "dr")
    for k, (value, off) in enumerate(want["dparams"]):
        near(dparams[k], value, 2 * off, f"vector {k}")


def both_ways(R, C, dtype, post, pre, vectors, seed=0, gap=0, shift=0):
    block, p, u, r, dout, dy = make(R, C, dtype, post, pre, vectors, seed)
    u, r, dout, dy = (matrix(a, gap, shift) for a in (u, r, dout, dy))
    none = torch.zeros(R, C, dtype=u.dtype, device="cuda")
    out, du, dr = (matrix(none, gap + 1, shift) for _ in range(3))
    y = matrix(none, gap, shift) if pre != "none" else None
    around = [(t, t._base.isnan().sum()) for t in (out, du, dr)]
    stats = torch.full((4, R), math.nan, device="cuda")
    q = dq.MxMatrix(R, C, "cuda") if pre != "none" else None
    dq.dqrm_residual_norm_fwd(block, u, r, out, y=y, stats=stats, q=q)
    check_forward(block, p, u, r, out, y, stats)
    if q is not None:  # the codes are those of the product's own quantisation, of y before its rounding: in 32 bits of y itself
        if dtype == "f32":
            same = dq.MxMatrix(R, C, "cuda")
            dq.dqrm_mxfp4_quant(y, same)
            assert torch.equal(q.codes, same.codes) and torch.equal(q.scales, same.scales)
        # without codes: many rows may lie over threads in another way then, and add up in another order
        out2, y2, stats2 = matrix(none, gap + 1, shift), matrix(none, gap, shift), torch.full((4, R), math.nan, device="cuda")
        dq.dqrm_residual_norm_fwd(block, u, r, out2, y=y2, stats=stats2)
        check_forward(block, p, u, r, out2, y2, stats2)
        again = torch.empty_like(out)
        dq.dqrm_residual_norm_fwd(block, u, r, again)
        assert torch.equal(again, out2)
    kept = torch.where(torch.isnan(stats), torch.tensor([0.0, 1.0, 0.0, 1.0], device="cuda")[:, None], stats)
    dparams = torch.full((5, C), math.nan, device="cuda")
    dq.dqrm_residual_norm_bwd(block, dout, dy, u, out, stats, du, dr, dparams, space(R, C))
    check_backward(p, dout, dy, u, out, kept, du, dr, dparams)
    assert all(t._base.isnan().sum() == n for t, n in around)
    # each output by itself
    for name, want in (("du", du), ("dr", dr)):
        got = torch.empty_like(want)
        dq.dqrm_residual_norm_bwd(block, dout, dy, u, out, stats, **{name: got})
        assert torch.equal(got, want)
    return block, u, r, out, y, stats, dout, dy, du, dr, dparams


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_shapes(shape, dtype):
    kinds = BOTH[(shape[0] + shape[1]) % 8]
    both_ways(*shape, dtype, "layer", "layer", True, seed=sum(shape))
    both_ways(*shape, dtype, *kinds, False, seed=sum(shape), gap=3, shift=1)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", MANY)
def test_many_rows(shape, dtype):
    """Rows over threads as many of them are; the columns' vectors in registers, in LDS and in memory."""
    both_ways(*shape, dtype, "layer", "rms", True, seed=sum(shape), gap=shape[1] % 3, shift=shape[1] % 2)
    both_ways(*shape, dtype, "rms", "layer", True, seed=sum(shape))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("post, pre", BOTH)
def test_kinds(post, pre, dtype):
    for cols, gap, shift in ((200, 0, 0), (1500, 5, 3)):
        for vectors in (False, True):
            both_ways(300, cols, dtype, post, pre, vectors, seed=cols, gap=gap, shift=shift)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("post, pre", BOTH)
@pytest.mark.parametrize("cols", [5, 300, 1001, 4500])
def test_in_place(post, pre, cols, dtype):
    """The residual stream's memory takes out, and the gradients' memory the gradients, as separate memory does."""
    block, p, u, r, dout, dy = make(260, cols, dtype, post, pre, True, 3)
    out, du, dr = torch.empty_like(u), torch.empty_like(u), torch.empty_like(u)
    stats = torch.ones(4, 260, device="cuda")
    dq.dqrm_residual_norm_fwd(block, u, r, out, stats=stats)
    dparams = torch.empty(5, cols, device="cuda")
    dq.dqrm_residual_norm_bwd(block, dout, dy, u, out, stats, du, dr, dparams, space(260, cols))
    for into in (r.clone(), u.clone()):
        first = into if torch.equal(into, u) else u
        dq.dqrm_residual_norm_fwd(block, first, r if first is into else into, into)
        assert torch.equal(into, out)
    for a, b in ((0, 1), (1, 0), (2, 3), (0, 2)):
        mem = [dout.clone(), dy.clone(), u.clone(), out.clone()]
        sums = torch.empty_like(dparams)
        dq.dqrm_residual_norm_bwd(block, *mem, stats, mem[a], mem[b], sums, space(260, cols))
        assert torch.equal(mem[a], du) and torch.equal(mem[b], dr) and torch.equal(sums, dparams)


@pytest.mark.parametrize("dtype", TYPES)
def test_without_a_gradient_of_the_residual_stream(dtype):
    block, p, u, r, dout, dy = make(70, 300, dtype, "rms", "layer", True, 4)
    out, stats = torch.empty_like(u), torch.empty(4, 70, device="cuda")
    dq.dqrm_residual_norm_fwd(block, u, r, out, stats=stats)
    results = []
    for d in (None, torch.zeros_like(dy)):
        du, dr, dparams = torch.empty_like(u), torch.empty_like(u), torch.empty(5, 300, device="cuda")
        dq.dqrm_residual_norm_bwd(block, d, dy, u, out, stats, du, dr, dparams, space(70, 300))
        results.append((du, dr, dparams))
    assert all(torch.equal(a, b) for a, b in zip(*results))


def test_no_rows_and_rows_that_are_not_finite():
    block, p, u, r, dout, dy = make(40, 200, "f32", "layer", "rms", True, 5)
    out, y, stats = torch.empty_like(u), torch.empty_like(u), torch.empty(4, 40, device="cuda")
    dq.dqrm_residual_norm_fwd(block, u[:0], r[:0], out[:0], y=y[:0], stats=stats[:, :0].contiguous())
    dparams = torch.full((5, 200), math.nan, device="cuda")
    dq.dqrm_residual_norm_bwd(block, dout[:0], dy[:0], u[:0], out[:0], stats[:, :0].contiguous(), None, None, dparams, space(0, 200))
    assert bool((dparams == 0).all())
    dq.dqrm_residual_norm_fwd(block, u, r, out, y=y, stats=stats)
    good = out.clone(), y.clone()
    u[7, 3], r[9, 0], u[11, 199] = math.inf, math.nan, -math.inf
    dq.dqrm_residual_norm_fwd(block, u, r, out, y=y, stats=stats)
    bad = torch.zeros(40, dtype=torch.bool, device="cuda")
    bad[[7, 9, 11]] = True
    assert torch.equal(out[~bad], good[0][~bad]) and torch.equal(y[~bad], good[1][~bad]) and bool(torch.isnan(y[bad]).all())


def test_a_row_of_equal_values():
    """No variance, with eps and without: the offset, or what 0 times an infinity is."""
    for eps, fine in ((1e-5, True), (0.0, False)):
        block = dq.ResidualNorm(post=dq.NORM_NONE, pre=dq.NORM_LAYER, pre_eps=eps)
        u, r = torch.full((3, 96), 1.0, device="cuda"), torch.full((3, 96), 2.0, device="cuda")
        out, y = torch.empty_like(u), torch.empty_like(u)
        dq.dqrm_residual_norm_fwd(block, u, r, out, y=y)
        assert bool((out == 3).all()) and bool((y == 0).all() if fine else torch.isnan(y).all())


def test_against_differences():
    block, p, u, r, dout, dy = make(5, 37, "f32", "layer", "layer", True, 6)
    out, stats = torch.empty_like(u), torch.empty(4, 5, device="cuda")
    dq.dqrm_residual_norm_fwd(block, u, r, out, stats=stats)
    du, dr, dparams = torch.empty_like(u), torch.empty_like(u), torch.empty(5, 37, device="cuda")
    dq.dqrm_residual_norm_bwd(block, dout, dy, u, out, stats, du, dr, dparams, space(5, 37))

    def value(args):
        q = dict(p, **{n: args[n] for n in ("post_gamma", "post_beta", "gate", "pre_gamma", "pre_beta")})
        w = ref.forward(q, args["u"], args["r"])
        return float((w["out"][0] * dout.double()).sum() + (w["y"][0] * dy.double()).sum())
    base = dict(u=u.double(), r=r.double(), **{n: p[n] for n in ("post_gamma", "post_beta", "gate", "pre_gamma", "pre_beta")})
    got = dict(u=du, r=dr, post_gamma=dparams[0], post_beta=dparams[1], gate=dparams[2], pre_gamma=dparams[3], pre_beta=dparams[4])
    gen = torch.Generator(device="cuda").manual_seed(2)
    for name, slope in got.items():
        way = torch.randn(base[name].shape, dtype=torch.float64, device="cuda", generator=gen)
        h = 1e-5
        up, down = (dict(base, **{name: base[name] + s * h * way}) for s in (1, -1))
        want = (value(up) - value(down)) / (2 * h)
        # (64-bit differences: h^2 and 2^-52 / h of the values, 1e-9; the gradients' 32 bits: 1e-5 of their sizes' sum is 80 u of it)
        assert abs(want - float((slope.double() * way).sum())) <= 1e-5 * float((slope.double().abs() * way.abs()).sum()), name


def test_captured_and_replayed():
    block, p, u, r, dout, dy = make(500, 1024, "bf16", "rms", "layer", True, 7)
    make_out = lambda: [torch.empty_like(u), torch.empty_like(u), torch.empty(4, 500, device="cuda"), torch.empty_like(u), torch.empty_like(u),  # noqa: E731
                        torch.empty(5, 1024, device="cuda"), space(500, 1024)]

    def step(o):
        dq.dqrm_residual_norm_fwd(block, u, r, o[0], y=o[1], stats=o[2])
        dq.dqrm_residual_norm_bwd(block, dout, dy, u, o[0], o[2], o[3], o[4], o[5], o[6])
    static, eager = make_out(), make_out()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(static)
    for _ in range(4):
        u.copy_(torch.randn_like(u))
        dy.copy_(torch.randn_like(u))
        graph.replay()
        torch.cuda.synchronize()
        step(eager)
        assert all(torch.equal(a, b) for a, b in zip(static[:6], eager[:6]))
