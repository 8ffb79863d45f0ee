"""The padding behind a row's values is part of the format, for rows that are not finite too: zero codes, and scale byte 0 for blocks
that hold no value, whichever way the row was laid over threads."""
import numpy as np
import pytest
import torch

import mx_reference as ref
from mx_reference import TYPES, f64, on_gpu

pytestmark = pytest.mark.gpu


def _dq():
    import paper_2410_20046_amd as dq

    return dq


# (a row in one thread's chunk, in parts of a wave, a wave, a workgroup, and read more than once; the last block full, in part and missing)
@pytest.mark.parametrize("rows", [6, 300])
@pytest.mark.parametrize("cols", [5, 9, 33, 64, 100, 200, 385, 700, 1030, 3000, 5000, 10000, 16300, 16400])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_norm_writes_the_padding_of_rows_that_are_not_finite(dtype, cols, rows):
    dq = _dq()
    print("padding", dtype, rows, cols, flush=True)
    x = np.random.default_rng(cols).standard_normal((rows, cols))
    x[0, cols // 2], x[1, cols - 1], x[2, 0] = np.nan, np.inf, -np.inf
    x[3] = 1.0  # no variance: with eps = 0 every value is 0 * inf
    x[4] = 0.0
    gamma, beta = torch.linspace(0.5, 2.0, cols, device="cuda"), torch.linspace(-1.0, 1.0, cols, device="cuda")
    for g, b in ((None, None), (gamma, beta)):
        q, y = dq.MxMatrix(rows, cols, "cuda"), torch.empty((rows, cols), dtype=TYPES[dtype], device="cuda")
        q.codes.fill_(0xA5), q.scales.fill_(0x5A)
        dq.dqrm_layernorm_fwd(on_gpu(x, TYPES[dtype]), g, b, 0.0, y=y, q=q)
        assert np.isnan(f64(y[:5])).all() and np.isfinite(f64(y[5:])).all()
        code, scale = ref.quantise(f64(y[:5]))
        np.testing.assert_array_equal(q.scales[:5].cpu().numpy(), scale)
        np.testing.assert_array_equal(q.codes[:5].cpu().numpy(), ref.pack(code))
        blocks, values = -(-cols // 32), -(-cols // 2)
        assert not q.scales[:, blocks:].any() and not q.codes[:, values:].any()
        assert (q.scales[5:, :blocks] != 255).all()


@pytest.mark.parametrize("rows", [2, 4, 7, 40])
@pytest.mark.parametrize("cols", [8, 200, 2000])
def test_linear_behind_a_norm_keeps_nans_to_their_rows(cols, rows):
    """Few rows, which the product normalises itself, and more: a row's NaNs stay its own."""
    dq = _dq()
    rng = np.random.default_rng(cols)
    x = rng.standard_normal((rows, cols)).astype(np.float32)
    x[rows // 2, cols - 1] = np.nan
    x[0] = 3.0  # (eps = 0)
    n = 70
    w = dq.MxMatrix(n, cols, "cuda")
    dq.dqrm_mxfp4_quant(torch.from_numpy(rng.standard_normal((n, cols))).float().cuda(), w)
    out = torch.empty((rows, n), device="cuda")
    ws = torch.empty(max(dq.dqrm_mxfp4_linear_workspace_bytes(rows, n, cols), 256), dtype=torch.uint8, device="cuda")
    dq.dqrm_mxfp4_linear(torch.from_numpy(x).cuda(), w, out, eps=0.0, workspace=ws)
    want = np.zeros(rows, bool)
    want[[0, rows // 2]] = True
    np.testing.assert_array_equal(np.isnan(f64(out)), np.repeat(want[:, None], n, 1))
