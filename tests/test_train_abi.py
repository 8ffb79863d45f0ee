"""CPU-only checks of the boundary of the residual norms, the softmax cross entropy and the gradients' clip: every refusal comes before
anything is launched, so none of these calls needs a GPU, and the binding refuses what the C calls cannot see."""
import ctypes as C

import pytest
import torch

import paper_2410_20046_amd as dq
from launches import would_launch

FAKE = 0x10000  # non-null, aligned, never dereferenced: validation fails first
BIG = 1 << 40
OK, INVALID, UNSUPPORTED, SMALL = dq.OK, dq.ERR_INVALID_ARG, dq.ERR_UNSUPPORTED, dq.ERR_WORKSPACE_TOO_SMALL
MOST = 2147482623
NAN, INF = float("nan"), float("inf")


def norm(post=dq.NORM_RMS, pre=dq.NORM_LAYER, pg=None, pb=None, gate=None, eg=None, eb=None, scale=1.0, post_eps=1e-5, pre_eps=1e-5):
    return C.byref(dq.dqrm_residual_norm_t(post, pre, pg, pb, gate, eg, eb, scale, post_eps, pre_eps))


def test_residual_norm_forward_refusals():
    L = dq.lib()

    def fwd(dtype=0, rows=8, cols=40, n="ok", u=FAKE, ldu=40, r=FAKE, ldr=40, out=FAKE, ldo=40, y=FAKE, ldy=40, stats=None, q=None):
        return L.dqrm_residual_norm_fwd(dtype, rows, cols, norm() if n == "ok" else n, u, ldu, r, ldr, out, ldo, y, ldy, stats, q, None)
    assert fwd(n=None) == INVALID and fwd(dtype=3) == INVALID and fwd(rows=-1) == INVALID and fwd(cols=0) == INVALID and fwd(cols=-1) == INVALID
    assert fwd(rows=MOST + 1) == UNSUPPORTED and fwd(cols=16385, ldu=BIG) == UNSUPPORTED
    for kinds in (dict(post=3), dict(post=-1), dict(pre=7)):
        assert fwd(n=norm(**kinds)) == INVALID
    for eps in (-1.0, NAN):
        assert fwd(n=norm(post_eps=eps)) == INVALID and fwd(n=norm(pre_eps=eps)) == INVALID
    assert fwd(n=norm(post=0, pg=FAKE)) == INVALID and fwd(n=norm(post=0, pb=FAKE)) == INVALID  # the gain of a norm that is not there
    assert fwd(n=norm(pre=0, eg=FAKE), y=None) == INVALID and fwd(n=norm(pre=0)) == INVALID  # y of a norm that is not there
    for name in ("pg", "pb", "gate", "eg", "eb"):
        assert fwd(n=norm(**{name: FAKE + 2})) == INVALID
    for name, ld in (("u", "ldu"), ("r", "ldr"), ("out", "ldo")):
        assert fwd(**{name: None}) == INVALID and fwd(**{name: FAKE + 2}) == INVALID and fwd(**{ld: 39}) == INVALID and fwd(**{ld: 2 * BIG}) == UNSUPPORTED
    assert fwd(y=FAKE + 1) == INVALID and fwd(ldy=39) == INVALID and fwd(stats=FAKE + 2) == INVALID
    assert fwd(dtype=1, u=FAKE + 1) == INVALID
    mx = lambda r, c, codes=FAKE: C.byref(dq.dqrm_mxfp4_t(r, c, codes, FAKE))  # noqa: E731
    assert fwd(q=mx(8, 41)) == INVALID and fwd(q=mx(8, 40, FAKE + 8)) == INVALID
    assert fwd(rows=0, u=None, r=None, out=None, y=None) == OK  # nothing to do


def test_residual_norm_backward_refusals():
    L = dq.lib()

    def bwd(dtype=0, rows=8, cols=40, n="ok", dout=FAKE, lddout=40, dy=FAKE, lddy=40, u=FAKE, ldu=40, out=FAKE, ldo=40, stats=FAKE, du=FAKE, lddu=40, dr=FAKE,
            lddr=40, dparams=FAKE, ws=FAKE, ws_bytes=1 << 30):
        return L.dqrm_residual_norm_bwd(dtype, rows, cols, norm() if n == "ok" else n, dout, lddout, dy, lddy, u, ldu, out, ldo, stats, du, lddu, dr, lddr, dparams,
                                        ws, ws_bytes, None)
    assert bwd(n=None) == INVALID and bwd(dtype=9) == INVALID and bwd(rows=-1) == INVALID and bwd(cols=16385) == UNSUPPORTED
    assert bwd(du=None, dr=None, dparams=None) == INVALID  # no output
    assert bwd(n=norm(pre=0), dout=None) == INVALID  # no gradient
    assert bwd(dy=None) == INVALID and bwd(out=None) == INVALID and bwd(u=None) == INVALID and bwd(stats=None) == INVALID
    assert bwd(stats=FAKE + 2) == INVALID and bwd(dparams=FAKE + 1) == INVALID
    for name in ("dout", "dy", "u", "out", "du", "dr"):
        assert bwd(**{name: FAKE + 2}) == INVALID and bwd(**{"ldo" if name == "out" else "ld" + name: 39}) == INVALID, name
    need = dq.dqrm_residual_norm_bwd_workspace_bytes(8, 40)
    assert need >= 4 * 40 * 4
    assert bwd(ws=None) == INVALID and bwd(ws=FAKE + 16) == INVALID and bwd(ws_bytes=need - 1) == SMALL
    assert dq.dqrm_residual_norm_bwd_workspace_bytes(-1, 40) == 0 and dq.dqrm_residual_norm_bwd_workspace_bytes(8, 16385) == 0


def test_loss_refusals():
    L = dq.lib()

    def fwd(dtype=0, m=8, v=50, k=40, x=FAKE, ldx=40, w=FAKE, ldw=40, bias=None, scale=1.0, targets=FAKE, loss=FAKE, lse=FAKE, ws=FAKE, ws_bytes=1 << 40):
        return L.dqrm_softmax_xent_fwd(dtype, m, v, k, x, ldx, w, ldw, bias, scale, targets, loss, lse, ws, ws_bytes, None)

    def bwd(dtype=0, m=8, v=50, k=40, x=FAKE, ldx=40, w=FAKE, ldw=40, bias=None, scale=1.0, targets=FAKE, lse=FAKE, grad=FAKE, dx=FAKE, lddx=40, dw=FAKE, lddw=40,
            dbias=FAKE, ws=FAKE, ws_bytes=1 << 40):
        return L.dqrm_softmax_xent_bwd(dtype, m, v, k, x, ldx, w, ldw, bias, scale, targets, lse, grad, dx, lddx, dw, lddw, dbias, ws, ws_bytes, None)
    for call in (fwd, bwd):
        assert call(dtype=3) == INVALID and call(m=-1) == INVALID and call(v=-1) == INVALID and call(k=-1) == INVALID and call(v=0) == INVALID
        assert call(m=MOST + 1) == UNSUPPORTED and call(v=MOST + 1) == UNSUPPORTED and call(k=(1 << 22) + 1, ldx=1 << 23, ldw=1 << 23) == UNSUPPORTED
        assert call(m=1 << 20, v=1 << 21) == UNSUPPORTED  # more tiles than 2^22
        assert call(x=None) == INVALID and call(w=None) == INVALID and call(x=FAKE + 2) == INVALID and call(w=FAKE + 2) == INVALID
        assert call(ldx=39) == INVALID and call(ldw=39) == INVALID
        assert call(ldx=(1 << 22) + 8) == UNSUPPORTED and call(ldw=(1 << 22) + 8) == UNSUPPORTED
        assert call(scale=NAN) == INVALID and call(scale=INF) == INVALID and call(bias=FAKE + 2) == INVALID
        assert call(targets=None) == INVALID and call(targets=FAKE + 4) == INVALID
        assert call(lse=None) == INVALID and call(lse=FAKE + 2) == INVALID
        assert call(ws=None) == INVALID and call(ws=FAKE + 16) == INVALID
    assert fwd(loss=None) == INVALID and fwd(loss=FAKE + 1) == INVALID
    assert bwd(grad=None) == INVALID and bwd(grad=FAKE + 2) == INVALID and bwd(dx=None, dw=None, dbias=None) == INVALID
    assert bwd(dx=FAKE + 2) == INVALID and bwd(dw=FAKE + 2) == INVALID and bwd(dbias=FAKE + 2) == INVALID and bwd(lddx=39) == INVALID and bwd(lddw=39) == INVALID
    need = dq.dqrm_softmax_xent_fwd_workspace_bytes(8, 50, 40, torch.float32)
    assert need > 0 and fwd(ws_bytes=need - 1) == SMALL
    need = dq.dqrm_softmax_xent_bwd_workspace_bytes(8, 50, 40, torch.float32)
    assert need > 0 and bwd(ws_bytes=need - 1) == SMALL
    for query in (L.dqrm_softmax_xent_fwd_workspace_bytes, L.dqrm_softmax_xent_bwd_workspace_bytes):
        assert query(-1, 5, 5, 0) == 0 and query(5, 5, (1 << 22) + 1, 0) == 0 and query(5, 5, 5, 7) == 0 and query(1 << 20, 1 << 21, 5, 0) == 0


def grads(*items):
    return (dq.dqrm_grad_t * max(len(items), 1))(*items)


def item(data=FAKE, rows=8, cols=40, ld=40, out=None, ld_out=0, count=None, dtype=0):
    return dq.dqrm_grad_t(data, rows, cols, ld, out, ld_out, count, dtype)


def test_gradient_refusals():
    L = dq.lib()

    def calls(*items, n=None, kind=0, norm_=FAKE, norms=None, ws=FAKE, ws_bytes=1 << 30, most=1.0):
        g, n = grads(*items), len(items) if n is None else n
        return {L.dqrm_grad_norm(g, n, kind, norm_, norms, ws, ws_bytes, None), L.dqrm_grad_clip(g, n, kind, most, norm_, norms, ws, ws_bytes, None)}
    assert calls(item(), n=-1) == {INVALID} and calls(item(), n=65537) == {UNSUPPORTED} and L.dqrm_grad_norm(None, 2, 0, FAKE, None, FAKE, 1 << 20, None) == INVALID
    assert calls(item(), kind=2) == {INVALID} and calls(item(), kind=-1) == {INVALID}
    assert calls(item(), norm_=None) == {INVALID} and calls(item(), norm_=FAKE + 2) == {INVALID} and calls(item(), norms=FAKE + 2) == {INVALID}
    for bad in (item(dtype=3), item(rows=-1), item(cols=-1), item(data=None), item(data=FAKE + 2), item(dtype=1, data=FAKE + 1), item(ld=39), item(out=FAKE + 2, ld_out=40),
                item(out=FAKE, ld_out=39), item(count=FAKE + 2)):
        assert calls(item(), bad) == {INVALID}
        assert L.dqrm_grad_scale(grads(bad), 1, FAKE, 1.0, None) == INVALID
        assert L.dqrm_grad_workspace_bytes(grads(bad), 1) == 0
    assert calls(item(rows=MOST + 1)) == {UNSUPPORTED} and calls(item(rows=1, cols=(1 << 40) + 1)) == {UNSUPPORTED}
    assert calls(item(rows=1 << 20, cols=1 << 25, ld=1 << 25)) == {UNSUPPORTED}
    assert calls(*[item(rows=1, cols=1 << 40, data=FAKE + (i << 43)) for i in range(17)]) == {UNSUPPORTED}  # 2^44 values in all
    need = L.dqrm_grad_workspace_bytes(grads(item()), 1)
    assert need > 0 and calls(item(), ws=None) == {INVALID} and calls(item(), ws=FAKE + 8) == {INVALID} and calls(item(), ws_bytes=need - 1) == {SMALL}
    for most in (-1.0, NAN):
        assert L.dqrm_grad_clip(grads(item()), 1, 0, most, FAKE, None, FAKE, 1 << 20, None) == INVALID
        assert L.dqrm_grad_scale(grads(item()), 1, FAKE, most, None) == INVALID
    assert L.dqrm_grad_scale(grads(item()), 1, None, 1.0, None) == INVALID and L.dqrm_grad_scale(grads(item()), 1, FAKE + 1, 1.0, None) == INVALID


def test_tensors_on_top_of_each_other_are_refused_where_they_are_written():
    L = dq.lib()
    size = 8 * 40 * 4
    scale = lambda *items: L.dqrm_grad_scale(grads(*items), len(items), FAKE, 1.0, None)  # noqa: E731
    clip = lambda *items: L.dqrm_grad_clip(grads(*items), len(items), 0, 1.0, FAKE, None, FAKE, 1 << 20, None)  # noqa: E731
    for call in (scale, clip):
        assert call(item(), item()) == INVALID  # the same one twice
        assert call(item(), item(data=FAKE + size - 4)) == INVALID
        assert call(item(data=FAKE + 4 * size), item(rows=1, cols=4000, ld=4000)) == INVALID
        assert call(item(), item(data=FAKE + 8 * size, out=FAKE, ld_out=40)) == INVALID  # an output on another tensor


def test_binding_refuses_what_the_calls_cannot_see():
    x, t = torch.zeros(4, 64), torch.zeros(4, dtype=torch.int64)
    with pytest.raises(AssertionError):
        dq.ResidualNorm(pre_gamma=torch.ones(64), gate=torch.ones(63))
    with pytest.raises(AssertionError):
        dq.dqrm_residual_norm_fwd(dq.ResidualNorm(gate=torch.ones(63)), x, x, x, stream=0)
    with pytest.raises(AssertionError):
        dq.dqrm_residual_norm_fwd(dq.ResidualNorm(), x, x.bfloat16(), x, stream=0)
    with pytest.raises(AssertionError):
        dq.dqrm_residual_norm_fwd(dq.ResidualNorm(), x, x, x, stats=torch.zeros(4, 5), stream=0)
    with pytest.raises(AssertionError):
        dq.dqrm_residual_norm_bwd(dq.ResidualNorm(), None, None, x, x, torch.zeros(4, 4), x)
    v = torch.zeros(4)
    with pytest.raises(AssertionError):
        dq.dqrm_softmax_xent_fwd(x, torch.zeros(9, 63), t, v, v)
    with pytest.raises(AssertionError):
        dq.dqrm_softmax_xent_fwd(x, torch.zeros(9, 64), t.int(), v, v)
    with pytest.raises(AssertionError):
        dq.dqrm_softmax_xent_fwd(x, torch.zeros(9, 64), t, torch.zeros(5), v)
    with pytest.raises(AssertionError):
        dq.dqrm_softmax_xent_bwd(x, torch.zeros(9, 64), t, v, v, dw=torch.zeros(8, 64))
    with pytest.raises(AssertionError):
        dq.Grads([x.double()])
    with pytest.raises(AssertionError):
        dq.Grads([torch.zeros(4, 6, 8).transpose(1, 2)])
    with pytest.raises(AssertionError):
        dq.Grads([x], out=[torch.zeros(4, 63)])
    with pytest.raises(AssertionError):
        dq.Grads([x], out=[])
    with pytest.raises(AssertionError):
        dq.Grads([x], counts={1: torch.zeros(1, dtype=torch.int32)})
    with pytest.raises(AssertionError):
        dq.Grads([x], counts={0: torch.zeros(1, dtype=torch.int64)})
    with pytest.raises(AssertionError):
        dq.dqrm_grad_norm(dq.Grads([x]), torch.zeros(2))
    with pytest.raises(dq.DqrmError) as e:
        dq.dqrm_grad_norm(dq.Grads([x]), torch.zeros(1))
    assert e.value.code == INVALID  # host memory


# ---- what would be launched ----------------------------------------------------------------------------------------------------

ROOM = 1 << 60


def xent_fwd(t, m, v, k, ws=ROOM):
    return ("dqrm_softmax_xent_fwd", t, m, v, k, FAKE, max(k, 1), FAKE, max(k, 1), FAKE, 1.0, FAKE, FAKE, FAKE, FAKE, ws, None)


def xent_bwd(t, m, v, k, ws=ROOM):
    return ("dqrm_softmax_xent_bwd", t, m, v, k, FAKE, max(k, 1), FAKE, max(k, 1), FAKE, 1.0, FAKE, FAKE, FAKE, FAKE, max(k, 1), FAKE, max(k, 1), FAKE, FAKE, ws, None)


@pytest.mark.parametrize("m, v, k", [(1, (1 << 30) - 3, 8), (1 << 28, 64, 40), (8, 4_000_000, 1024), (64, 1 << 22, 513), (1 << 20, 100_000, 16), (3, 7, 1 << 22)])
def test_large_losses_are_launched(m, v, k):
    """Grids stay below 2^32 threads, whatever the number of rows, classes and pieces of them."""
    for t in (0, 1, 2):
        for rc, launches in would_launch([xent_fwd(t, m, v, k), xent_bwd(t, m, v, k)]):
            assert rc == OK and launches
            assert all(not l.failed and max(l.grid[i] * l.block[i] for i in range(3)) < 1 << 32 for l in launches)


@pytest.mark.parametrize("v, k", [(1, 1), (1000, 16), (50021, 1021), (200003, 64), (131072, 4096), (12, 8192), (1_000_000, 512)])
@pytest.mark.parametrize("m", [64, 1000, 8192, 20000])
def test_the_workspace_of_the_loss_is_enough_for_fewer_rows(m, v, k):
    some = sorted({1, 2, 8, 9, 16, 17, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 513, 1023, 2047, m // 3, m // 2, m - 1, m})
    some = [s for s in some if 1 <= s <= m]
    for t in (0, 1, 2):
        (forward, _), (backward, _) = would_launch([("dqrm_softmax_xent_fwd_workspace_bytes", m, v, k, t), ("dqrm_softmax_xent_bwd_workspace_bytes", m, v, k, t)])
        calls = [xent_fwd(t, s, v, k, forward) for s in some] + [xent_bwd(t, s, v, k, backward) for s in some]
        assert {rc for rc, _ in would_launch(calls)} == {OK}


def resnorm(rows, cols):
    return [("dqrm_residual_norm_bwd_workspace_bytes", rows, cols)]


@pytest.mark.parametrize("cols", [1, 7, 40, 300, 1200, 4100, 8192, 16384])
def test_the_workspace_of_the_residual_norm_is_enough_for_fewer_rows(cols):
    rows = [1, 2, 31, 32, 33, 100, 255, 257, 5000, 100000]
    sizes = [n for n, _ in would_launch([resnorm(r, cols)[0] for r in rows])]
    assert sizes == sorted(sizes)
