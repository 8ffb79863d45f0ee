"""The next item of a history: INT4 embedding tables, residual blocks, a softmax over all items, gradients clipped together.

    python examples/next_item.py [--steps 200] [--batch 1024] [--items 20000] [--dim 64] [--blocks 2]

A sample is a bag of items that somebody has looked at; the model says which one comes next.  The history's table is looked up and pooled with
INT4 rows; residual blocks (two linear layers with a ReLU between them, in torch) are joined by dqrm_residual_norm_fwd, which normalises the block's
output, adds it gated to the stream and normalises the sum for the next block; dqrm_softmax_xent_fwd takes the loss over the whole table of
items without its logits in memory.  Backward, all gradients, the history table's sparse ones among them, are clipped by their common norm
before the tables' INT8 update and the step of everything else.
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2410_20046_amd as dq  # noqa: E402


def byte_buffer(n: int) -> torch.Tensor:
    return torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")


class Block:
    """u = relu(y W1^T) W2^T, joined with the stream r: r' = r + gate N1(u), y' = N2(r')."""

    def __init__(self, batch: int, dim: int, gen: torch.Generator):
        empty = lambda *s: torch.empty(*s, device="cuda")  # noqa: E731
        self.w1 = torch.randn(2 * dim, dim, device="cuda", generator=gen) * dim ** -0.5
        self.w2 = torch.randn(dim, 2 * dim, device="cuda", generator=gen) * (2 * dim) ** -0.5
        one, zero = torch.ones(dim, device="cuda"), torch.zeros(dim, device="cuda")
        self.vectors = torch.stack((one, zero, 0.5 * one, one, zero))  # gains and offsets of both norms around the gate, as the gradients come
        post_gamma, post_beta, gate, pre_gamma, pre_beta = self.vectors
        self.norm = dq.ResidualNorm(post=dq.NORM_RMS, pre=dq.NORM_LAYER, post_gamma=post_gamma, post_beta=post_beta, gate=gate, pre_gamma=pre_gamma, pre_beta=pre_beta)
        self.out, self.next_y, self.stats = empty(batch, dim), empty(batch, dim), empty(4, batch)
        self.du, self.dr, self.dvectors = empty(batch, dim), empty(batch, dim), empty(5, dim)
        self.dw1, self.dw2 = torch.empty_like(self.w1), torch.empty_like(self.w2)
        self.ws = byte_buffer(dq.dqrm_residual_norm_bwd_workspace_bytes(batch, dim))

    def forward(self, r, y):
        self.y, self.h = y, torch.relu(y @ self.w1.t())
        self.u = self.h @ self.w2.t()
        dq.dqrm_residual_norm_fwd(self.norm, self.u, r, self.out, y=self.next_y, stats=self.stats)
        return self.out, self.next_y

    def backward(self, dout, dy):
        """Gradients of the stream behind the block (or None) and of its normalised form -> those in front of it."""
        dq.dqrm_residual_norm_bwd(self.norm, dout, dy, self.u, self.out, self.stats, self.du, self.dr, self.dvectors, self.ws)
        torch.mm(self.du.t(), self.h, out=self.dw2)
        dh = (self.du @ self.w2) * (self.h > 0)
        torch.mm(dh.t(), self.y, out=self.dw1)
        return self.dr, dh @ self.w1


class NextItem:
    def __init__(self, batch: int, items: int, dim: int, blocks: int, history: int = 8, seed: int = 0):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.B, self.V, self.D, self.history = batch, items, dim, history
        empty = lambda *s: torch.empty(*s, device="cuda")  # noqa: E731
        self.tables = dq.Tables(np.array([0, items], dtype=np.int64), dim, torch.randn(items, dim, device="cuda", generator=gen) * 0.5,
                                torch.empty(items, dim // 2, dtype=torch.uint8, device="cuda"))
        dq.dqrm_find_scale(self.tables)
        dq.dqrm_pack_int4(self.tables)
        self.bufs = dq.StepBuffers(1, dim, batch, batch * history, torch.device("cuda"))
        self.offsets = torch.arange(batch + 1, dtype=torch.int64, device="cuda") * history
        self.gamma, self.beta = torch.ones(dim, device="cuda"), torch.zeros(dim, device="cuda")
        self.y0, self.mean, self.rstd = empty(batch, dim), empty(batch), empty(batch)
        self.dx0, self.dgamma, self.dbeta = empty(batch, dim), empty(dim), empty(dim)
        self.blocks = [Block(batch, dim, gen) for _ in range(blocks)]
        self.w_items = torch.randn(items, dim, device="cuda", generator=gen) * dim ** -0.5
        self.b_items = torch.zeros(items, device="cuda")
        self.dw_items, self.db_items = empty(items, dim), empty(items)
        self.loss, self.lse, self.dy = empty(batch), empty(batch), empty(batch, dim)
        self.ws = byte_buffer(max(dq.dqrm_softmax_xent_fwd_workspace_bytes(batch, items, dim, torch.float32),
                                  dq.dqrm_softmax_xent_bwd_workspace_bytes(batch, items, dim, torch.float32), dq.dqrm_layernorm_bwd_workspace_bytes(batch, dim)))
        b = self.bufs
        self.parameters = [self.gamma, self.beta, self.w_items, self.b_items] + [p for k in self.blocks for p in (k.w1, k.w2, k.vectors)]
        self.gradients = [self.dgamma, self.dbeta, self.dw_items, self.db_items] + [g for k in self.blocks for g in (k.dw1, k.dw2, k.dvectors)]
        # the history table's gradient has as many rows as the batch has items, a number that stays on the GPU; its largest magnitude, which the
        # update takes its scale from, is scaled with it
        self.all = dq.Grads(self.gradients + [b.values], counts={len(self.gradients): b.num_unique})
        self.largest = dq.Grads([b.g_absmax])
        self.norm, self.norm_ws = empty(1), byte_buffer(dq.dqrm_grad_workspace_bytes(self.all))

    def forward(self, idx: torch.Tensor, targets: torch.Tensor) -> torch.Tensor:
        """The rows' losses; a negative target: none."""
        dq.dqrm_embbag_fwd(self.tables, idx, self.offsets, self.B, dq.FWD_PACKED, self.bufs.out)
        r = self.bufs.out.view(self.B, self.D)
        dq.dqrm_layernorm_fwd(r, self.gamma, self.beta, 1e-5, y=self.y0, mean=self.mean, rstd=self.rstd)
        y = self.y0
        for block in self.blocks:
            r, y = block.forward(r, y)
        self.y = y
        dq.dqrm_softmax_xent_fwd(y, self.w_items, targets, self.loss, self.lse, bias=self.b_items, workspace=self.ws)
        return self.loss

    def backward(self, idx: torch.Tensor, targets: torch.Tensor) -> torch.Tensor:
        """All gradients of the mean loss; returns that of the pooled history."""
        grad = (targets >= 0) / (targets >= 0).sum().clamp(min=1)
        dq.dqrm_softmax_xent_bwd(self.y, self.w_items, targets, self.lse, grad, dx=self.dy, dw=self.dw_items, dbias=self.db_items, bias=self.b_items,
                                 workspace=self.ws)
        dr, dy = None, self.dy
        for block in reversed(self.blocks):
            dr, dy = block.backward(dr, dy)
        x = self.bufs.out.view(self.B, self.D)
        dq.dqrm_layernorm_bwd(dy, x, self.mean, self.rstd, self.gamma, self.dx0, self.dgamma, self.dbeta, self.ws)
        self.dpooled = self.dx0 if dr is None else self.dx0 + dr
        b = self.bufs
        dq.dqrm_embbag_bwd(self.tables, idx, self.offsets, self.B, self.dpooled.view(self.B, 1, self.D), b.sorted_pos, b.uniq_rows, b.seg_offsets,
                           b.table_uniq_offsets, b.num_unique, b.values, b.g_absmax, b.workspace)
        return self.dpooled

    def clip(self, max_norm: float) -> None:
        dq.dqrm_grad_clip(self.all, max_norm, self.norm, workspace=self.norm_ws)
        dq.dqrm_grad_scale(self.largest, self.norm, max_norm)

    def step(self, lr: float) -> None:
        for p, g in zip(self.parameters, self.gradients):
            p.add_(g, alpha=-lr)
        b = self.bufs
        dq.dqrm_grad_quant_int8(1, self.D, b.cap, b.values, b.table_uniq_offsets, b.g_absmax, b.gq, b.g_scale)
        dq.dqrm_sparse_update(self.tables, b.cap, b.uniq_rows, b.table_uniq_offsets, b.gq, b.g_scale, lr)


def samples(model: NextItem, gen: torch.Generator):
    """Histories within one of 50 groups of items, the next item from the same group; one row in 16 has no target."""
    group = torch.randint(0, 50, (model.B, 1), device="cuda", generator=gen)
    items = (torch.randint(0, model.V // 50, (model.B, model.history + 1), device="cuda", generator=gen) * 50 + group).clamp(max=model.V - 1)
    targets = torch.where(torch.rand(model.B, device="cuda", generator=gen) < 1 / 16, -1, items[:, -1])
    return items[:, :-1].reshape(-1).contiguous(), targets.contiguous()


def run(steps: int = 200, batch: int = 1024, items: int = 20000, dim: int = 64, blocks: int = 2, lr: float = 1.0, max_norm: float = 1.0, say=print):
    """(mean loss of the first step, of the last)"""
    model = NextItem(batch, items, dim, blocks)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    losses = []
    for k in range(steps):
        idx, targets = samples(model, gen)
        loss = model.forward(idx, targets)
        losses.append(loss.sum() / (targets >= 0).sum())
        model.backward(idx, targets)
        model.clip(max_norm)
        model.step(lr)
        if k % 50 == 0 or k == steps - 1:
            say(f"step {k}: loss {float(losses[-1]):.4f}, gradients' norm {float(model.norm):.4f}")
    code, table, value = dq.dqrm_check_status()
    assert code == 0, (code, table, value)
    return float(losses[0]), float(losses[-1])


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("steps", 200), ("batch", 1024), ("items", 20000), ("dim", 64), ("blocks", 2)):
        ap.add_argument("--" + name, type=int, default=value)
    for name, value in (("lr", 1.0), ("max-norm", 1.0)):
        ap.add_argument("--" + name, type=float, default=value)
    run(**{k.replace("-", "_"): v for k, v in vars(ap.parse_args()).items()})
