"""A click model with a 4-bit top MLP: INT4 embedding tables, layer norms, linear layers whose operands are MXFP4.

    python examples/mxfp4_top_mlp.py [--steps 200] [--batch 2048] [--hidden 512,256] [--dtype bf16]

Trains on synthetic samples, then serves single samples.  A layer of the MLP is y = relu(norm(x) W^T + b): forward, the norm writes
MXFP4 codes and statistics, and the product reads the codes; backward, the gradient behind the ReLU goes to MXFP4 both ways from one read
(with the bias's gradient), two products give the input's and the weights' gradients (straight-through: the weights that the step goes to
are FP32), and the norm's backward ends the layer.  A request takes one call per layer.  torch holds memory and does the loss and the SGD
step of the MLP; the tables take their step in the library.
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2410_20046_amd as dq  # noqa: E402

EPS = 1e-5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def byte_buffer(n: int) -> torch.Tensor:
    return torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")


class NormLinear:
    """norm, 4-bit linear layer, ReLU if asked: its parameters, and the buffers of one batch size."""

    def __init__(self, batch: int, fan_in: int, fan_out: int, relu: bool, dtype: torch.dtype, gen: torch.Generator):
        M, N, K = batch, fan_out, fan_in
        empty = lambda *s, t=torch.float32: torch.empty(*s, dtype=t, device="cuda")  # noqa: E731
        self.relu = relu
        self.w = torch.randn(N, K, device="cuda", generator=gen) * (2.0 / K) ** 0.5
        self.b, self.gamma, self.beta = (torch.zeros(N, device="cuda"), torch.ones(K, device="cuda"), torch.zeros(K, device="cuda"))
        self.dw, self.db, self.dgamma, self.dbeta = empty(N, K), empty(N), empty(K), empty(K)
        self.w_q, self.w_t = dq.MxMatrix(N, K, "cuda"), dq.MxMatrix(K, N, "cuda")
        self.x_q, self.x_t = dq.MxMatrix(M, K, "cuda"), dq.MxMatrix(K, M, "cuda")
        self.g_q, self.g_t = dq.MxMatrix(M, N, "cuda"), dq.MxMatrix(N, M, "cuda")
        self.xn, self.mean, self.rstd = empty(M, K, t=dtype), empty(M), empty(M)
        self.y, self.dxn, self.dx = empty(M, N, t=dtype), empty(M, K, t=dtype), empty(M, K, t=dtype)
        self.ws = byte_buffer(max(dq.dqrm_mxfp4_matmul_workspace_bytes(M, N, K), dq.dqrm_mxfp4_matmul_workspace_bytes(M, K, N),
                                  dq.dqrm_mxfp4_matmul_workspace_bytes(N, K, M), dq.dqrm_mxfp4_quant_workspace_bytes(M, N),
                                  dq.dqrm_layernorm_bwd_workspace_bytes(M, K), dq.dqrm_mxfp4_linear_workspace_bytes(M, N, K)))
        self.quantise_weights()

    def quantise_weights(self) -> None:
        dq.dqrm_mxfp4_quant(self.w, self.w_q, self.w_t)

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        self.x = x
        dq.dqrm_layernorm_fwd(x, self.gamma, self.beta, EPS, y=self.xn, mean=self.mean, rstd=self.rstd, q=self.x_q)
        dq.dqrm_mxfp4_matmul(self.x_q, self.w_q, self.y, bias=self.b, relu=self.relu, workspace=self.ws)
        return self.y

    def backward(self, dy: torch.Tensor) -> torch.Tensor:
        dq.dqrm_mxfp4_quant(dy, self.g_q, self.g_t, gate=self.y if self.relu else None, col_sums=self.db, workspace=self.ws)
        dq.dqrm_mxfp4_quant(self.xn, None, self.x_t)
        dq.dqrm_mxfp4_matmul(self.g_q, self.w_t, self.dxn, workspace=self.ws)
        dq.dqrm_mxfp4_matmul(self.g_t, self.x_t, self.dw, workspace=self.ws)
        dq.dqrm_layernorm_bwd(self.dxn, self.x, self.mean, self.rstd, self.gamma, self.dx, self.dgamma, self.dbeta, self.ws)
        return self.dx

    def step(self, lr: float) -> None:
        for p, g in ((self.w, self.dw), (self.b, self.db), (self.gamma, self.dgamma), (self.beta, self.dbeta)):
            p.add_(g, alpha=-lr)
        self.quantise_weights()

    def serve(self, x: torch.Tensor) -> torch.Tensor:
        out = torch.empty(x.shape[0], self.w_q.rows, dtype=x.dtype, device="cuda")
        dq.dqrm_mxfp4_linear(x, self.w_q, out, bias=self.b, relu=self.relu, gamma=self.gamma, beta=self.beta, eps=EPS, workspace=self.ws)
        return out


class ClickModel:
    def __init__(self, batch: int, hidden, tables: int = 8, rows: int = 1000, dim: int = 16, dense: int = 13, dtype=torch.bfloat16, seed: int = 0):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.B, self.T, self.D, self.dense, self.dtype = batch, tables, dim, dense, dtype
        master = torch.randn(tables * rows, dim, device="cuda", generator=gen) * 0.1
        packed = torch.empty(tables * rows, dim // 2, dtype=torch.uint8, device="cuda")
        self.tables = dq.Tables(np.arange(tables + 1, dtype=np.int64) * rows, dim, master, packed)
        dq.dqrm_find_scale(self.tables)
        dq.dqrm_pack_int4(self.tables)
        self.bufs = dq.StepBuffers(tables, dim, batch, tables * batch, torch.device("cuda"))
        self.offsets = torch.arange(tables * batch + 1, dtype=torch.int64, device="cuda")
        widths = [dense + tables * dim] + list(hidden) + [1]
        self.layers = [NormLinear(batch, i, o, k + 2 < len(widths), dtype, gen) for k, (i, o) in enumerate(zip(widths[:-1], widths[1:]))]

    def features(self, dense: torch.Tensor, idx: torch.Tensor) -> torch.Tensor:
        """The tables' rows (one per table and sample) behind the dense features."""
        b, n = self.bufs, dense.shape[0]
        out = b.out if n == self.B else torch.empty(n, self.T, self.D, device="cuda")
        offsets = self.offsets if n == self.B else torch.arange(self.T * n + 1, dtype=torch.int64, device="cuda")
        dq.dqrm_embbag_fwd(self.tables, idx, offsets, n, dq.FWD_PACKED, out)
        return torch.cat([dense, out.view(n, -1)], 1).to(self.dtype)

    def train_step(self, dense: torch.Tensor, idx: torch.Tensor, labels: torch.Tensor, lr: float) -> torch.Tensor:
        x = self.features(dense, idx)
        for layer in self.layers:
            x = layer.forward(x)
        z = x.float()[:, 0]
        loss = torch.nn.functional.softplus(z).mean() - (z * labels).mean()
        g = ((torch.sigmoid(z) - labels) / self.B).to(self.dtype)[:, None].contiguous()
        for layer in reversed(self.layers):
            g = layer.backward(g)
        for layer in self.layers:
            layer.step(lr)
        b = self.bufs
        grad_out = g[:, self.dense:].float().reshape(self.B, self.T, self.D).contiguous()
        dq.dqrm_embbag_bwd(self.tables, idx, self.offsets, self.B, grad_out, b.sorted_pos, b.uniq_rows, b.seg_offsets, b.table_uniq_offsets, b.num_unique,
                           b.values, b.g_absmax, b.workspace)
        dq.dqrm_grad_quant_int8(self.T, self.D, b.cap, b.values, b.table_uniq_offsets, b.g_absmax, b.gq, b.g_scale)
        dq.dqrm_sparse_update(self.tables, b.cap, b.uniq_rows, b.table_uniq_offsets, b.gq, b.g_scale, lr)
        return loss

    def serve(self, dense: torch.Tensor, idx: torch.Tensor) -> torch.Tensor:
        x = self.features(dense, idx)
        for layer in self.layers:
            x = layer.serve(x)
        return torch.sigmoid(x.float()[:, 0])


def samples(model: ClickModel, rng: torch.Generator, secret: torch.Tensor):
    """Dense features, one row number per table (table-major), and clicks that go by the features and by the first table's rows."""
    dense = torch.randn(model.B, model.dense, device="cuda", generator=rng)
    idx = torch.randint(0, 1000, (model.T, model.B), device="cuda", generator=rng)
    clicks = (dense @ secret + (idx[0] % 2) * 2.0 - 1.0 > 0).float()
    return dense, idx.reshape(-1), clicks


def run(steps: int = 200, batch: int = 2048, hidden=(512, 256), dtype: str = "bf16", lr: float = 0.1, say=print):
    """(loss of the first steps, loss of the last steps, largest difference between served and trained-forward probabilities)"""
    model = ClickModel(batch, hidden, dtype=TYPES[dtype])
    rng = torch.Generator(device="cuda")
    rng.manual_seed(1)
    secret = torch.randn(model.dense, device="cuda", generator=rng)
    losses = []
    for k in range(steps):
        losses.append(model.train_step(*samples(model, rng, secret), lr))
        if k % 50 == 0 or k == steps - 1:
            say(f"step {k}: loss {float(losses[-1]):.4f}")
    dense, idx, _ = samples(model, rng, secret)
    x = model.features(dense, idx)
    for layer in model.layers:
        x = layer.forward(x)
    want = torch.sigmoid(x.float()[:, 0])
    worst = 0.0
    for k in sorted({0, min(1, batch - 1), batch // 2, batch - 1}):  # requests of one sample
        got = model.serve(dense[k:k + 1], idx.view(model.T, batch)[:, k].contiguous())
        worst = max(worst, float((got[0] - want[k]).abs()))
    got = model.serve(dense[:5], idx.view(model.T, batch)[:, :5].contiguous().reshape(-1))
    worst = max(worst, float((got - want[:5]).abs().max()))
    code, table, value = dq.dqrm_check_status()
    assert code == 0, (code, table, value)
    n = max(1, min(10, steps // 4))
    first, last = (float(torch.stack(l).mean()) for l in (losses[:n], losses[-n:]))
    say(f"loss {first:.4f} -> {last:.4f}; requests differ from the batch by at most {worst:.2e}")
    return first, last, worst


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--batch", type=int, default=2048)
    ap.add_argument("--hidden", default="512,256")
    ap.add_argument("--dtype", choices=sorted(TYPES), default="bf16")
    ap.add_argument("--lr", type=float, default=0.1)
    a = ap.parse_args()
    run(a.steps, a.batch, [int(w) for w in a.hidden.split(",")], a.dtype, a.lr)
