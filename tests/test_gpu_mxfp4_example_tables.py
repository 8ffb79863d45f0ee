"""The 4-bit click model's step of its tables: their INT8 gradients, as the rows' segment sums are."""
import os
import sys

import numpy as np
import pytest
import torch

import paper_2410_20046_amd as dq

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("batch", [1, 64, 1000])
def test_a_step_moves_the_rows_by_their_gradients(batch):
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import mxfp4_top_mlp
    finally:
        sys.path.pop(0)
    model = mxfp4_top_mlp.ClickModel(batch, (40,))
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    samples = mxfp4_top_mlp.samples(model, gen, torch.randn(model.dense, device="cuda", generator=gen))
    master, lr = model.tables.master.clone(), 0.5
    model.train_step(*samples, lr)
    b = model.bufs
    n, ends = int(b.num_unique), b.table_uniq_offsets.cpu().numpy()
    assert n > 0 and float(b.values[:n].abs().max()) > 0
    table = torch.from_numpy(np.repeat(np.arange(model.T), np.diff(ends))).cuda()
    most = torch.stack([b.values[ends[t]:ends[t + 1]].abs().max() for t in range(model.T)]).double()
    # a scale is the table's largest magnitude over 127 (1e-8 at least), a gradient is off by half of one, and the update rounds twice
    scale = (most / 127).clamp(min=1e-8)
    assert bool(((b.g_scale.double() - scale).abs() <= 2.0 ** -22 * scale).all())
    rows = b.uniq_rows[:n] + table * (len(master) // model.T)  # (they are numbered in their tables)
    moved = (model.tables.master - master).double()
    want = torch.zeros_like(moved)
    want[rows] = -lr * b.values[:n].double()
    off = torch.zeros_like(moved)
    off[rows] = (lr * (0.501 * scale)[table])[:, None] + 2.0 ** -22 * master.double().abs()[rows]
    assert bool(((moved - want).abs() <= off).all()), float(((moved - want).abs() - off).max())
    assert dq.dqrm_check_status()[0] == 0
