"""The residual norms, the loss over many classes and the clip as they are used together: the example's gradients against 64-bit automatic
differentiation, its clip and its update."""
import math
import os
import sys

import pytest
import torch

import paper_2410_20046_amd as dq

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import next_item  # noqa: E402

pytestmark = pytest.mark.gpu


def plain(model, pooled, targets):
    """The mean loss and its gradients in 64 bits: of the pooled history and of the model's parameters."""
    x = pooled.double().clone().requires_grad_()
    p = [v.double().clone().requires_grad_() for v in model.parameters]
    gamma, beta, w, b = p[:4]
    layer = lambda v, g, o: (v - v.mean(1, keepdim=True)) / (v.var(1, unbiased=False, keepdim=True) + 1e-5).sqrt() * g + o  # noqa: E731
    r, y = x, layer(x, gamma, beta)
    for k in range(len(model.blocks)):
        w1, w2, vectors = p[4 + 3 * k:7 + 3 * k]
        u = torch.relu(y @ w1.t()) @ w2.t()
        n1 = u / ((u * u).mean(1, keepdim=True) + 1e-5).sqrt() * vectors[0] + vectors[1]
        r = r + vectors[2] * n1
        y = layer(r, vectors[3], vectors[4])
    l = y @ w.t() + b
    have = targets >= 0
    loss = (torch.logsumexp(l, 1) - l.gather(1, targets.clamp(min=0)[:, None])[:, 0])[have].mean()
    loss.backward()
    return float(loss.detach()), x.grad, [v.grad for v in p]


@pytest.mark.parametrize("batch, items, dim, blocks", [(64, 500, 16, 1), (300, 3001, 64, 2), (33, 700, 40, 0)])
def test_gradients_and_their_clip(batch, items, dim, blocks):
    model = next_item.NextItem(batch, items, dim, blocks, seed=3)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(batch)
    idx, targets = next_item.samples(model, gen)
    loss = model.forward(idx, targets)
    pooled = model.bufs.out.view(batch, dim).clone()
    dpooled = model.backward(idx, targets)
    want_loss, want_pooled, want = plain(model, pooled, targets)
    # 32-bit sums of up to some thousand terms in a chain of ten operations: 1e-5 of a gradient's norm is 84 roundings on top of each other
    assert abs(float(loss.sum() / (targets >= 0).sum()) - want_loss) <= 1e-5 * want_loss
    for got, w in zip([dpooled] + model.gradients, [want_pooled] + want):
        assert float((got.double() - w).norm()) <= 1e-5 * float(w.norm()) + 1e-12
    b = model.bufs
    n = int(b.num_unique)
    rows = b.values[:n].clone()
    total = math.sqrt(sum(float(g.double().square().sum()) for g in model.gradients) + float(rows.double().square().sum()))
    behind = b.values[n:].clone()
    before = [g.clone() for g in model.gradients]
    most, master = b.g_absmax.clone(), model.tables.master.clone()
    weights = [p.clone() for p in model.parameters]
    model.clip(total / 4)
    assert abs(float(model.norm) - total) <= 1e-7 * total
    for old, new in zip(before + [rows, most], model.gradients + [b.values[:n], b.g_absmax]):
        assert float((new.double() - old.double() / 4).norm()) <= 3e-7 * float(old.double().norm())
    assert torch.equal(b.values[n:].nan_to_num(5.0), behind.nan_to_num(5.0))
    model.step(0.5)
    for old, new, g in zip(weights, model.parameters, model.gradients):
        assert torch.equal(new, old.add(g, alpha=-0.5))
    # the update went to the history's rows, by its INT8 gradients: at most half a step of their scale from the clipped ones
    moved = (model.tables.master - master).double()
    want = torch.zeros_like(moved)
    want[b.uniq_rows[:n]] = -0.5 * b.values[:n].double()
    assert float((moved - want).abs().max()) <= 0.5 * float(b.g_scale[0]) * 0.5 * 1.001 + 1e-7 * float(master.abs().max())
    assert float(b.g_scale[0]) <= float(most[0]) / 4 / 127 * 1.001
    assert dq.dqrm_check_status()[0] == 0


def test_the_example_runs():
    first, last = next_item.run(steps=5, batch=200, items=1000, dim=32, say=lambda line: None)
    assert math.isfinite(first) and math.isfinite(last)


def test_the_step_captured_beside_eager_work():
    """Forward, backward and clip of one batch in a graph, replayed between eager steps of another model with the same buffers' sizes."""
    make = lambda: next_item.NextItem(128, 900, 32, 1, seed=4)  # noqa: E731
    static, eager = make(), make()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(9)
    idx, targets = next_item.samples(static, gen)

    def all_of_it(model, idx, targets):
        dq.dqrm_embbag_fwd(model.tables, idx, model.offsets, model.B, dq.FWD_PACKED, model.bufs.out)
        block = model.blocks[0]
        r = model.bufs.out.view(model.B, model.D)
        dq.dqrm_residual_norm_fwd(block.norm, r, r, block.out, y=block.next_y, stats=block.stats)
        dq.dqrm_softmax_xent_fwd(block.next_y, model.w_items, targets, model.loss, model.lse, bias=model.b_items, workspace=model.ws)
        dq.dqrm_softmax_xent_bwd(block.next_y, model.w_items, targets, model.lse, model.loss, dx=model.dy, dw=model.dw_items, dbias=model.db_items,
                                 bias=model.b_items, workspace=model.ws)
        dq.dqrm_residual_norm_bwd(block.norm, None, model.dy, r, block.out, block.stats, block.du, block.dr, block.dvectors, block.ws)
        dq.dqrm_grad_clip(model.some, 0.25, model.norm, workspace=model.norm_ws)
        return [model.loss, model.dy, model.dw_items, model.db_items, block.du, block.dr, block.dvectors, model.norm]
    for m in (static, eager):
        b = m.blocks[0]
        m.some = dq.Grads([m.dw_items, m.db_items, b.dvectors, b.du])
    s_idx, s_targets = idx.clone(), targets.clone()
    all_of_it(static, s_idx, s_targets)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = all_of_it(static, s_idx, s_targets)
    for _ in range(4):
        idx, targets = next_item.samples(eager, gen)
        s_idx.copy_(idx)
        s_targets.copy_(targets)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, all_of_it(eager, idx, targets)))
