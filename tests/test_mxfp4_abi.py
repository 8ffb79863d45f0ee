"""CPU-only checks of the layer norm's and the MXFP4 calls' boundary: every refusal comes before anything is launched, so none of these
calls needs a GPU, and the binding refuses what the C calls cannot see."""
import ctypes as C

import pytest
import torch

import paper_2410_20046_amd as dq
from paper_2410_20046_amd.binding import dqrm_mxfp4_t

FAKE = 0x1000  # non-null, aligned, never dereferenced: validation fails first
BIG = 1 << 40
INVALID, UNSUPPORTED, SMALL = dq.ERR_INVALID_ARG, dq.ERR_UNSUPPORTED, dq.ERR_WORKSPACE_TOO_SMALL
MOST = 2147482623


def q(rows, cols, codes=FAKE, scales=FAKE):
    return C.byref(dqrm_mxfp4_t(rows, cols, codes, scales))


def test_quant_refusals():
    L = dq.lib()

    def quant(dtype=0, rows=8, cols=40, x=FAKE, ldx=40, gate=None, ldgate=0, by_rows="ok", by_cols=None, sums=None, ws=None, ws_bytes=0):
        return L.dqrm_mxfp4_quant(dtype, rows, cols, x, ldx, gate, ldgate, q(rows, cols) if by_rows == "ok" else by_rows, by_cols, sums, ws, ws_bytes, None)
    assert quant(dtype=3) == INVALID and quant(dtype=-1) == INVALID
    assert quant(rows=-1) == INVALID and quant(cols=-1) == INVALID
    assert quant(rows=MOST + 1) == UNSUPPORTED and quant(cols=MOST + 1, ldx=BIG) == UNSUPPORTED
    assert quant(by_rows=None) == INVALID  # no output
    assert quant(x=None) == INVALID and quant(x=FAKE + 2) == INVALID and quant(dtype=1, x=FAKE + 1) == INVALID
    assert quant(ldx=39) == INVALID and quant(ldx=0) == INVALID and quant(ldx=-40) == INVALID and quant(ldx=BIG * 2) == UNSUPPORTED
    assert quant(gate=FAKE + 2, ldgate=40) == INVALID and quant(gate=FAKE, ldgate=39) == INVALID
    assert quant(by_rows=q(8, 41)) == INVALID and quant(by_rows=q(7, 40)) == INVALID
    assert quant(by_rows=q(8, 40, codes=None)) == INVALID and quant(by_rows=q(8, 40, scales=None)) == INVALID
    assert quant(by_rows=q(8, 40, codes=FAKE + 8)) == INVALID and quant(by_rows=q(8, 40, scales=FAKE + 2)) == INVALID
    assert quant(by_cols=q(8, 40)) == INVALID  # not the transposed shape
    assert quant(by_cols=q(40, 8, codes=FAKE + 4)) == INVALID
    assert quant(sums=FAKE + 2, ws=FAKE, ws_bytes=1 << 20) == INVALID
    need = dq.dqrm_mxfp4_quant_workspace_bytes(8, 40)
    assert need >= 40 * 4
    assert quant(sums=FAKE) == INVALID and quant(sums=FAKE, ws=FAKE + 16, ws_bytes=1 << 20) == INVALID
    assert quant(sums=FAKE, ws=FAKE, ws_bytes=need - 1) == SMALL
    assert dq.dqrm_mxfp4_quant_workspace_bytes(-1, 4) == 0 and dq.dqrm_mxfp4_quant_workspace_bytes(4, MOST + 1) == 0


def test_dequant_refusals():
    L = dq.lib()
    f = lambda m, dtype=0, out=FAKE, ldo=40: L.dqrm_mxfp4_dequant(m, dtype, out, ldo, None)  # noqa: E731
    assert f(None) == INVALID and f(q(8, 40), dtype=5) == INVALID
    assert f(q(-1, 40)) == INVALID and f(q(8, MOST + 1)) == UNSUPPORTED
    assert f(q(8, 40, codes=None)) == INVALID and f(q(8, 40, scales=FAKE + 1)) == INVALID
    assert f(q(8, 40), out=None) == INVALID and f(q(8, 40), out=FAKE + 1) == INVALID and f(q(8, 40), ldo=39) == INVALID


def test_matmul_refusals():
    L = dq.lib()

    def mm(a="ok", b="ok", bias=None, dtype=0, out=FAKE, ldo=30, ws=FAKE, ws_bytes=1 << 40):
        return L.dqrm_mxfp4_matmul(q(20, 64) if a == "ok" else a, q(30, 64) if b == "ok" else b, bias, 0, dtype, out, ldo, ws, ws_bytes, None)
    assert mm(a=None) == INVALID and mm(b=None) == INVALID
    assert mm(a=q(20, 65)) == INVALID  # inner sizes differ
    assert mm(a=q(-1, 64)) == INVALID and mm(a=q(MOST + 1, 64)) == UNSUPPORTED and mm(a=q(20, MOST + 1), b=q(30, MOST + 1)) == UNSUPPORTED
    assert mm(a=q(20, 64, codes=None)) == INVALID and mm(b=q(30, 64, codes=FAKE + 8)) == INVALID and mm(b=q(30, 64, scales=FAKE + 1)) == INVALID
    assert mm(dtype=3) == INVALID and mm(bias=FAKE + 1) == INVALID
    assert mm(out=None) == INVALID and mm(out=FAKE + 1) == INVALID and mm(ldo=29) == INVALID
    # a product that is cut along k needs its workspace
    need = dq.dqrm_mxfp4_matmul_workspace_bytes(20, 30, 65536)
    long = dict(a=q(20, 65536), b=q(30, 65536))
    if need:
        assert mm(**long, ws=None) == INVALID and mm(**long, ws=FAKE + 16) == INVALID and mm(**long, ws_bytes=need - 1) == SMALL
    assert dq.dqrm_mxfp4_matmul_workspace_bytes(-1, 4, 4) == 0 and dq.dqrm_mxfp4_matmul_workspace_bytes(4, 4, MOST + 1) == 0


def test_linear_refusals():
    L = dq.lib()

    def lin(dtype=0, m=4, x=FAKE, ldx=64, norm=0, gamma=None, beta=None, eps=1e-5, w="ok", bias=None, out=FAKE, ldo=30, ws=FAKE, ws_bytes=1 << 40):
        return L.dqrm_mxfp4_linear(dtype, m, x, ldx, norm, gamma, beta, eps, q(30, 64) if w == "ok" else w, bias, 0, out, ldo, ws, ws_bytes, None)
    assert lin(w=None) == INVALID and lin(w=q(30, 64, codes=None)) == INVALID and lin(w=q(-1, 64)) == INVALID
    assert lin(dtype=9) == INVALID and lin(m=-1) == INVALID and lin(m=MOST + 1) == UNSUPPORTED
    assert lin(x=None) == INVALID and lin(x=FAKE + 2) == INVALID and lin(ldx=63) == INVALID
    assert lin(out=None) == INVALID and lin(out=FAKE + 2) == INVALID and lin(ldo=29) == INVALID and lin(bias=FAKE + 2) == INVALID
    assert lin(gamma=FAKE) == INVALID and lin(beta=FAKE) == INVALID  # a gain without a norm
    assert lin(norm=1, gamma=FAKE + 2) == INVALID and lin(norm=1, eps=-1.0) == INVALID and lin(norm=1, eps=float("nan")) == INVALID
    need = dq.dqrm_mxfp4_linear_workspace_bytes(4, 30, 64)
    if need:
        assert lin(ws=None) == INVALID and lin(ws=FAKE + 8) == INVALID and lin(ws_bytes=need - 1) == SMALL
    assert dq.dqrm_mxfp4_linear_workspace_bytes(4, -1, 4) == 0


def test_norm_refusals():
    L = dq.lib()

    def fwd(dtype=0, rows=8, cols=40, x=FAKE, ldx=40, gamma=None, beta=None, eps=1e-5, y=FAKE, ldy=40, mean=None, rstd=None, m=None):
        return L.dqrm_layernorm_fwd(dtype, rows, cols, x, ldx, gamma, beta, eps, y, ldy, mean, rstd, m, None)
    assert fwd(dtype=3) == INVALID and fwd(rows=-1) == INVALID and fwd(cols=0) == INVALID and fwd(cols=MOST + 1) == UNSUPPORTED
    assert fwd(y=None) == INVALID  # no output
    assert fwd(x=None) == INVALID and fwd(x=FAKE + 1) == INVALID and fwd(ldx=39) == INVALID and fwd(ldy=39) == INVALID and fwd(y=FAKE + 2) == INVALID
    assert fwd(eps=-1e-9) == INVALID and fwd(eps=float("nan")) == INVALID
    assert fwd(gamma=FAKE + 1) == INVALID and fwd(beta=FAKE + 1) == INVALID and fwd(mean=FAKE + 2) == INVALID and fwd(rstd=FAKE + 2) == INVALID
    assert fwd(m=q(8, 41)) == INVALID and fwd(m=q(8, 40, codes=FAKE + 8)) == INVALID

    def bwd(dtype=0, rows=8, cols=40, dy=FAKE, lddy=40, x=FAKE, ldx=40, mean=FAKE, rstd=FAKE, gamma=None, dx=FAKE, lddx=40, dg=FAKE, db=FAKE, ws=FAKE, ws_bytes=1 << 30):
        return L.dqrm_layernorm_bwd(dtype, rows, cols, dy, lddy, x, ldx, mean, rstd, gamma, dx, lddx, dg, db, ws, ws_bytes, None)
    assert bwd(dtype=3) == INVALID and bwd(rows=-1) == INVALID and bwd(cols=0) == INVALID and bwd(rows=MOST + 1) == UNSUPPORTED
    assert bwd(dg=None) == INVALID and bwd(db=None) == INVALID and bwd(dx=None, dg=None, db=None) == INVALID
    assert bwd(dy=None) == INVALID and bwd(x=None) == INVALID and bwd(mean=None) == INVALID and bwd(rstd=None) == INVALID
    assert bwd(lddy=39) == INVALID and bwd(ldx=39) == INVALID and bwd(lddx=39) == INVALID and bwd(dx=FAKE + 2) == INVALID
    assert bwd(gamma=FAKE + 2) == INVALID and bwd(dg=FAKE + 2) == INVALID
    need = dq.dqrm_layernorm_bwd_workspace_bytes(8, 40)
    assert need >= 2 * 40 * 4
    assert bwd(ws=None) == INVALID and bwd(ws=FAKE + 16) == INVALID and bwd(ws_bytes=need - 1) == SMALL
    assert dq.dqrm_layernorm_bwd_workspace_bytes(8, -1) == 0


def test_binding_refuses_what_the_calls_cannot_see():
    x = torch.zeros(4, 64)
    with pytest.raises(AssertionError):
        dq.MxMatrix(4, 64, codes=torch.zeros(4, 32, dtype=torch.uint8))  # rows are padded to 128 values
    with pytest.raises(AssertionError):
        dq.dqrm_mxfp4_quant(x.t(), dq.MxMatrix(64, 4))  # a row's elements are not contiguous
    with pytest.raises(AssertionError):
        dq.dqrm_mxfp4_quant(x.double(), dq.MxMatrix(4, 64))
    with pytest.raises(AssertionError):
        dq.dqrm_mxfp4_quant(x, dq.MxMatrix(4, 64), gate=torch.zeros(4, 64, dtype=torch.bfloat16))
    with pytest.raises(AssertionError):
        dq.dqrm_layernorm_fwd(x, torch.ones(63), None, 1e-5, y=x)
    with pytest.raises(AssertionError):
        dq.dqrm_layernorm_bwd(x, x, torch.zeros(4), torch.zeros(5), None, x)
    with pytest.raises(AssertionError):
        dq.dqrm_mxfp4_matmul(dq.MxMatrix(4, 64), dq.MxMatrix(5, 64), torch.zeros(4, 4))
    with pytest.raises(dq.DqrmError) as e:
        dq.dqrm_mxfp4_quant(torch.zeros(1, 64).expand(4, 64), dq.MxMatrix(4, 64), stream=0)  # rows on top of each other
    assert e.value.code == dq.ERR_INVALID_ARG
