"""The end of a training step as timed cases with their plain forms: residual joins with their norms, the softmax cross entropy
over many classes, and the clip of all gradients by their norm.

  resnorm  out = res_scale r + gate N1(u), y = N2(out): u a block's output, r the residual stream, N1 the norm behind the block, N2
           the one before the next block (layer norm, RMS norm or none; gains, offsets and the gate are vectors over the columns).
           Forward with both norms' statistics, or (train) the backward with the gradients of u, r and all five vectors
  xent     l = scale x w^T + bias, lse = log of the sum of exp(l) over the classes, loss = lse - l[target]: forward, or
           (train) forward and backward: the gradients of x, w and bias for a given gradient of the rows' losses.
           A row whose target is negative has loss 0 and no gradient; a bias of -infinity takes a class out
  clip     the 2-norm (or the largest magnitude) of many gradient tensors together and of each, and the tensors times max_norm / norm where
           the norm is above max_norm.  Of a tensor with a count only the first `count` rows are there (a table's sparse gradient)
"""
from __future__ import annotations

import math
import random
from typing import List

import torch

own = False  # the package's operators instead of the plain forms

EPS = 1e-5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
MOST_FLOPS = 6 * 8192 * 131072 * 4096  # of a loss with its gradients
MOST_VALUES = 16384 * 8192             # of a matrix that is normalised
MOST_GRADS = 1 << 30                   # values of all gradient tensors together
PIECE = 1 << 30                        # logits that the plain form has at a time


def listed() -> List[dict]:
    return [
        # one request scored against the smallest configuration's table: all latency
        dict(name="xent one row", kind="xent", train=False, rows=1, classes=1000, width=16, dtype="f32", bias=False, scale=1.0),
        # evaluation of a few requests over an item table of wide rows: the table's bytes
        dict(name="xent few rows", kind="xent", train=False, rows=16, classes=200003, width=1024, dtype="bf16", bias=True, scale=1.0),
        # a small training batch over the same kind of table: bytes of the table, read and written
        dict(name="xent train few rows", kind="xent", train=True, rows=64, classes=131072, width=2048, dtype="bf16", bias=True, scale=1.0),
        # the Terabyte workload's batch and embedding width over a table of its larger ones, tables in 32 bits, a temperature
        dict(name="xent train item table", kind="xent", train=True, rows=8192, classes=200003, width=64, dtype="f32", bias=True, scale=4.0),
        # the matrix instructions' rate: a large batch, wide rows
        dict(name="xent train wide", kind="xent", train=True, rows=8192, classes=131072, width=4096, dtype="bf16", bias=False, scale=1.0),
        # odd sizes throughout, rows of a width that no vector divides
        dict(name="xent odd half", kind="xent", train=True, rows=2001, classes=50021, width=1021, dtype="f16", bias=True, scale=1.0),
        # the gradients of the Kaggle model's MLPs, one tensor a weight or bias, and a table's sparse ones: launches
        dict(name="clip kaggle", kind="clip", tensors=13, values=650000, dtype="f32", sparse=True, largest=False),
        # all gradients of a large model, most in 16 bits, from vectors to large matrices: bytes
        dict(name="clip large", kind="clip", tensors=400, values=MOST_GRADS, dtype="mixed", sparse=False, largest=False),
        # one token, between two blocks: latency
        dict(name="resnorm one row", kind="resnorm", train=False, rows=1, cols=4096, dtype="bf16", post="rms", pre="rms"),
        # a training batch's activations, forward and backward
        dict(name="resnorm wide", kind="resnorm", train=False, rows=16384, cols=8192, dtype="bf16", post="layer", pre="layer"),
        dict(name="resnorm bwd wide", kind="resnorm", train=True, rows=16001, cols=4096, dtype="bf16", post="rms", pre="rms"),
        # the Terabyte workload's batch at the MLPs' width, in 32 bits, no norm behind the block
        dict(name="resnorm bwd layer", kind="resnorm", train=True, rows=8192, cols=512, dtype="f32", post="none", pre="layer"),
    ]


def _log_int(rng, lo: int, hi: int) -> int:
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng) -> dict:
    kind = rng.choice(["xent", "xent", "clip", "resnorm"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    if kind == "clip":
        tensors = _log_int(rng, 1, 400)
        return dict(kind=kind, tensors=tensors, values=_log_int(rng, 64 * tensors, MOST_GRADS >> 2), dtype=rng.choice(["f32", "bf16", "f16", "mixed"]),
                    sparse=rng.random() < 0.5, largest=rng.random() < 0.3)
    if kind == "resnorm":
        cols = _log_int(rng, 8, 8192)
        post, pre = rng.choice([("none", "layer"), ("none", "rms"), ("layer", "none"), ("rms", "none"), ("layer", "layer"), ("rms", "rms"), ("layer", "rms")])
        return dict(kind=kind, train=rng.random() < 0.5, rows=_log_int(rng, 1, min(65536, MOST_VALUES // (2 * cols))), cols=cols, dtype=dtype, post=post, pre=pre)
    train = rng.random() < 0.6
    classes, width = _log_int(rng, 8, 1 << 20), _log_int(rng, 8, 8192)
    width = max(8, min(width, (1 << 29) // classes))
    most = MOST_FLOPS // (48 if dtype == "f32" else 4) // (6 if train else 2) // (classes * width)
    return dict(kind=kind, train=train, rows=_log_int(rng, 1, max(1, min(16384, most))), classes=classes, width=width, dtype=dtype,
                bias=rng.random() < 0.5, scale=rng.choice([1.0, 1.0, 0.125, 4.0]))


# ---- inputs ---------------------------------------------------------------------------------------------------------


def _normal(g, *shape) -> torch.Tensor:
    return torch.randn(*shape, device="cuda", dtype=torch.float32, generator=g)


def _gradients(g, rows: int, cols: int) -> torch.Tensor:
    """Small, of very different sizes from sample to sample; one sample in 16 has none."""
    size = 1e-3 * torch.exp(1.5 * _normal(g, rows, 1)) * (torch.rand(rows, 1, device="cuda", generator=g) > 1 / 16)
    return _normal(g, rows, cols) * size


def _sizes(case: dict) -> List[tuple]:
    """(rows, columns, type) of the gradient tensors: matrices and vectors whose sizes span a factor of some thousand."""
    rng = random.Random(case["tensors"] * 1000003 + case["values"])
    share = [math.exp(rng.uniform(0, 8)) for _ in range(case["tensors"])]
    out = []
    for k, s in enumerate(share):
        n = max(1, int(case["values"] * s / sum(share)))
        cols = 64 if case["sparse"] and k == 0 else n if rng.random() < 0.3 else min(n, _log_int(rng, 16, 8192))
        t = case["dtype"] if case["dtype"] != "mixed" else rng.choice(["bf16", "bf16", "bf16", "f16", "f32"])
        out.append((max(1, n // cols), cols, t))
    return out


def _views(sizes: List[tuple], of=TYPES):
    """The tensors one behind the other in a buffer of zeros for each type, as a program keeps its gradients."""
    room = {t: sum(r * c for r, c, is_of in sizes if is_of == t) for t in TYPES}
    flat = {t: torch.zeros(n, dtype=of[t], device="cuda") for t, n in room.items() if n}
    at, views = dict.fromkeys(TYPES, 0), []
    for r, c, t in sizes:
        views.append(flat[t][at[t]:at[t] + r * c].view(r, c))
        at[t] += r * c
    return list(flat.values()), views


def prepare(case: dict, seed: int) -> dict:
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    kind = case["kind"]
    s = dict(case=case)
    empty = lambda *shape, dtype=torch.float32: torch.empty(*shape, dtype=dtype, device="cuda")  # noqa: E731
    if kind == "clip":
        s["flat"], s["grads"] = _views(_sizes(case))
        s["out_flat"], s["out"] = _views(_sizes(case))
        for k, v in enumerate(s["grads"]):
            v.copy_(_normal(g, *v.shape) * math.exp(random.Random(seed + k).uniform(-9, -5)))
        s["norm"], s["norms"] = empty(1), empty(len(s["grads"]))
        s["count"] = None
        if case["sparse"]:  # the first tensor's rows behind the count hold what an earlier batch left there
            s["count"] = torch.tensor([s["grads"][0].shape[0] * 3 // 4], dtype=torch.int32, device="cuda")
        # (a norm that most steps exceed a little)
        values = sum(v.numel() for v in s["grads"])
        s["max_norm"] = 1e-3 if case["largest"] else 5e-4 * math.sqrt(values)
        return s
    t = TYPES[case["dtype"]]
    if kind == "resnorm":
        R, C = case["rows"], case["cols"]
        s["u"] = (_normal(g, R, C) * torch.exp(0.5 * _normal(g, 1, C)) + 0.3 * _normal(g, 1, C)).to(t)
        s["r"] = (_normal(g, R, C) * torch.exp(0.3 * _normal(g, R, 1))).to(t)
        for name in ("post", "pre"):
            s[name + "_gamma"] = 1 + 0.2 * _normal(g, C) if case[name] != "none" else None
            s[name + "_beta"] = 0.1 * _normal(g, C) if case[name] == "layer" else None
        s["gate"], s["res_scale"] = 0.5 + 0.2 * _normal(g, C), 0.875
        s["out"], s["stats"] = empty(R, C, dtype=t), torch.zeros(4, R, device="cuda")
        if not case["train"]:
            s["y"] = empty(R, C, dtype=t) if case["pre"] != "none" else None
            return s
        out, _, stats = _resnorm(s)  # what the forward has kept
        s["out"], s["stats"] = out.to(t), stats
        del s["r"]
        s["dout"] = _gradients(g, R, C).to(t)
        s["dy"] = _gradients(g, R, C).to(t) if case["pre"] != "none" else None
        s["du"], s["dr"], s["dparams"] = empty(R, C, dtype=t), empty(R, C, dtype=t), empty(5, C)
        return s
    M, V, K = case["rows"], case["classes"], case["width"]
    s["x"] = _normal(g, M, K).to(t)
    s["w"] = (_normal(g, V, K) * (1.5 / math.sqrt(K) / case["scale"])).to(t)
    s["targets"] = torch.randint(0, V, (M,), device="cuda", generator=g)
    s["bias"] = None
    if case["bias"]:  # classes' log popularity; some classes are not offered
        s["bias"] = _normal(g, V)
        s["bias"][(torch.rand(V, device="cuda", generator=g) < 1 / 64).index_fill(0, s["targets"], False)] = -math.inf
    if M > 1:  # rows without a target: padding
        s["targets"][torch.rand(M, device="cuda", generator=g) < 1 / 16] = -1
    s["loss"], s["lse"] = empty(M), empty(M)
    if case["train"]:
        have = s["targets"] >= 0
        s["grad"] = have / have.sum().clamp(min=1)
        s["dx"], s["dw"], s["dbias"] = empty(M, K, dtype=t), empty(V, K, dtype=t), empty(V)
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------


def _norm(kind, v, gamma, beta):
    """(normalised, mean, rstd) in 32 bits"""
    if kind == "none":
        return v, torch.zeros_like(v[:, 0]), torch.zeros_like(v[:, 0])
    mean = v.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(v[:, :1])
    d = v - mean
    rstd = 1.0 / torch.sqrt((d * d).mean(1, keepdim=True) + EPS)
    out = d * rstd * gamma
    return (out if beta is None else out + beta), mean[:, 0], rstd[:, 0]


def _resnorm(s: dict):
    v, m1, r1 = _norm(s["case"]["post"], s["u"].float(), s["post_gamma"], s["post_beta"])
    out = s["res_scale"] * s["r"].float() + s["gate"] * v
    y, m2, r2 = _norm(s["case"]["pre"], out, s["pre_gamma"], s["pre_beta"])
    return out, y, torch.stack((m1, r1, m2, r2))


def _norm_bwd(kind, dy, v, mean, rstd, gamma):
    """(gradient of v, of the gain, of the offset)"""
    z = (v - mean[:, None]) * rstd[:, None]
    by_z = dy * gamma
    d = by_z - z * (by_z * z).mean(1, keepdim=True)
    if kind == "layer":
        d = d - by_z.mean(1, keepdim=True)
    return d * rstd[:, None], (dy * z).sum(0), dy.sum(0)


def _plain_resnorm(s: dict):
    case = s["case"]
    t = TYPES[case["dtype"]]
    if not case["train"]:
        out, y, stats = _resnorm(s)
        return dict(out=out.to(t), stats=stats, **({} if case["pre"] == "none" else dict(y=y.to(t))))
    u, g = s["u"].float(), s["dout"].float()
    m1, r1, m2, r2 = s["stats"]
    zero = torch.zeros(case["cols"], device="cuda")
    pre_gamma, pre_beta, post_gamma, post_beta = zero, zero, zero, zero
    if case["pre"] != "none":
        d, pre_gamma, pre_beta = _norm_bwd(case["pre"], s["dy"].float(), s["out"].float(), m2, r2, s["pre_gamma"])
        g = g + d
    h, v = g * s["gate"], u
    du = h
    if case["post"] != "none":
        v = (u - m1[:, None]) * r1[:, None] * s["post_gamma"]
        v = v if s["post_beta"] is None else v + s["post_beta"]
        du, post_gamma, post_beta = _norm_bwd(case["post"], h, u, m1, r1, s["post_gamma"])
    dparams = torch.stack((post_gamma, post_beta, (g * v).sum(0), pre_gamma, pre_beta))
    return dict(du=du.to(t), dr=(s["res_scale"] * g).to(t), dparams=dparams)


def _logits(x, w, bias, scale):
    l = (x @ w.t()) * scale
    return l if bias is None else l + bias


def _plain_xent(s: dict):
    case = s["case"]
    x, w, bias, scale, targets = s["x"].float(), s["w"].float(), s["bias"], case["scale"], s["targets"]
    M, V = case["rows"], case["classes"]
    step = max(1, min(V, PIECE // M))
    pieces = [(a, min(a + step, V)) for a in range(0, V, step)]
    top = torch.full((M,), -math.inf, device="cuda")
    total = torch.zeros(M, device="cuda")
    at_target = torch.zeros(M, device="cuda")
    for a, b in pieces:
        l = _logits(x, w[a:b], None if bias is None else bias[a:b], scale)
        new = torch.maximum(top, l.amax(1))
        total = total * torch.exp(top - new) + torch.exp(l - new[:, None]).sum(1)
        top = new
        here = (targets >= a) & (targets < b)
        at_target = torch.where(here, l.gather(1, (targets - a).clamp(0, b - a - 1)[:, None])[:, 0], at_target)
    lse = top + torch.log(total)
    loss = torch.where(targets >= 0, lse - at_target, torch.zeros_like(lse))
    if not case["train"]:
        return dict(loss=loss, lse=lse)
    t = TYPES[case["dtype"]]
    grad = torch.where(targets >= 0, s["grad"], torch.zeros_like(s["grad"]))
    dx = torch.zeros_like(x)
    dw, dbias = torch.empty_like(s["w"]), torch.empty(V, device="cuda")
    for a, b in pieces:
        if len(pieces) > 1:
            l = _logits(x, w[a:b], None if bias is None else bias[a:b], scale)
        d = torch.exp(l - lse[:, None])
        here = ((targets >= a) & (targets < b)).nonzero()[:, 0] if len(pieces) > 1 else (targets >= 0).nonzero()[:, 0]
        d[here, targets[here] - a] -= 1.0
        d *= grad[:, None]
        dx += d @ w[a:b]
        dw[a:b] = ((d.t() @ x) * scale).to(t)
        dbias[a:b] = d.sum(0)
    return dict(loss=loss, lse=lse, dx=(dx * scale).to(t), dw=dw, dbias=dbias)


def _live(s: dict) -> List[torch.Tensor]:
    """The tensors, of the one that has a count the rows that are there."""
    if s["count"] is None:
        return s["grads"]
    first = s["grads"][0]
    there = torch.arange(first.shape[0], device="cuda") < s["count"]
    return [torch.where(there[:, None], first, torch.zeros_like(first))] + s["grads"][1:]


def _plain_clip(s: dict):
    live = _live(s)
    if s["case"]["largest"]:
        norms = torch.stack([v.float().abs().amax() for v in live])
        norm = norms.amax()
    else:
        squares = torch.stack([(v.float() ** 2).sum() for v in live])
        norms, norm = torch.sqrt(squares), torch.sqrt(squares.sum())
    c = torch.where(norm > s["max_norm"], s["max_norm"] / norm, torch.ones_like(norm))
    for v, out in zip(live, s["out"]):
        out.copy_(v.float() * c)
    return dict(norm=norm[None], norms=norms, out=s["out_flat"])


def _plain(s: dict):
    return {"xent": _plain_xent, "clip": _plain_clip, "resnorm": _plain_resnorm}[s["case"]["kind"]](s)


def _own(s: dict):
    import paper_2410_20046_amd as dq

    case = s["case"]
    kind = case["kind"]
    byte = lambda n: torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")  # noqa: E731
    norms = {"none": dq.NORM_NONE, "layer": dq.NORM_LAYER, "rms": dq.NORM_RMS}
    if "plan" not in s:  # the descriptors and the workspace that a program makes once and keeps
        p = s["plan"] = dict(ws=None, bwd_ws=None)
        if kind == "clip":
            p["grads"] = dq.Grads(s["grads"], out=s["out"], counts={0: s["count"]} if case["sparse"] else None)
            p["ws"] = byte(dq.dqrm_grad_workspace_bytes(p["grads"]))
        elif kind == "xent":
            t, shape = s["x"].dtype, (case["rows"], case["classes"], case["width"])
            p["ws"] = byte(dq.dqrm_softmax_xent_fwd_workspace_bytes(*shape, t))
            if case["train"]:
                p["bwd_ws"] = byte(dq.dqrm_softmax_xent_bwd_workspace_bytes(*shape, t))
        else:
            p["block"] = dq.ResidualNorm(post=norms[case["post"]], pre=norms[case["pre"]], post_gamma=s["post_gamma"], post_beta=s["post_beta"],
                                         gate=s["gate"], pre_gamma=s["pre_gamma"], pre_beta=s["pre_beta"], res_scale=s["res_scale"], post_eps=EPS, pre_eps=EPS)
            if case["train"]:
                p["ws"] = byte(dq.dqrm_residual_norm_bwd_workspace_bytes(case["rows"], case["cols"]))
    p = s["plan"]
    if kind == "clip":
        dq.dqrm_grad_clip(p["grads"], s["max_norm"], s["norm"], kind=dq.GRAD_NORM_MAX if case["largest"] else dq.GRAD_NORM_2, norms=s["norms"], workspace=p["ws"])
        return dict(norm=s["norm"], norms=s["norms"], out=s["out_flat"])
    if kind == "xent":
        dq.dqrm_softmax_xent_fwd(s["x"], s["w"], s["targets"], s["loss"], s["lse"], bias=s["bias"], scale=case["scale"], workspace=p["ws"])
        out = dict(loss=s["loss"], lse=s["lse"])
        if case["train"]:
            dq.dqrm_softmax_xent_bwd(s["x"], s["w"], s["targets"], s["lse"], s["grad"], dx=s["dx"], dw=s["dw"], dbias=s["dbias"], bias=s["bias"],
                                     scale=case["scale"], workspace=p["bwd_ws"])
            out.update(dx=s["dx"], dw=s["dw"], dbias=s["dbias"])
        return out
    if not case["train"]:
        dq.dqrm_residual_norm_fwd(p["block"], s["u"], s["r"], s["out"], y=s["y"], stats=s["stats"])
        return dict(out=s["out"], stats=s["stats"], **({} if s["y"] is None else dict(y=s["y"])))
    dq.dqrm_residual_norm_bwd(p["block"], s["dout"], s["dy"], s["u"], s["out"], s["stats"], s["du"], s["dr"], dparams=s["dparams"], workspace=p["ws"])
    return dict(du=s["du"], dr=s["dr"], dparams=s["dparams"])


def run(state: dict):
    return _own(state) if own else _plain(state)


# ---- what a pass cannot do without ----------------------------------------------------------------------------------


def work(case: dict) -> dict:
    if case["kind"] == "clip":
        sizes = _sizes(case)
        return dict(bytes=sum(2 * r * c * (4 if t == "f32" else 2) for r, c, t in sizes), flops=3 * sum(r * c for r, c, _ in sizes))
    size = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "resnorm":
        R, C = case["rows"], case["cols"]
        matrices = (3 if case["pre"] == "none" else 4) + (2 if case["train"] and case["pre"] != "none" else 1 if case["train"] else 0)
        return dict(bytes=matrices * R * C * size + 16 * R + (40 if case["train"] else 20) * C, flops=(40 if case["train"] else 20) * R * C)
    M, V, K = case["rows"], case["classes"], case["width"]
    # (train: the logits once and the two gradients' products; an implementation that keeps no logits computes them twice)
    times = 2 if case["train"] else 1
    return dict(bytes=times * (M + V) * K * size + (4 * V * times if case["bias"] else 0) + 16 * M, flops=(6 if case["train"] else 2) * M * V * K)


# ---- the same from the definitions in 64 bits -----------------------------------------------------------------------


def _exact_norm(kind, v, gamma, beta):
    if kind == "none":
        nothing = v.new_zeros(v.shape[0])
        return v, nothing, nothing
    mean = v.sum(1) / v.shape[1] if kind == "layer" else v.new_zeros(v.shape[0])
    centred = v - mean[:, None]
    rstd = (centred.square().sum(1) / v.shape[1] + EPS) ** -0.5
    out = centred * rstd[:, None] * gamma.double()
    return (out + beta.double() if beta is not None else out), mean, rstd


def _exact_resnorm(s: dict):
    case = s["case"]
    if not case["train"]:
        v, m1, r1 = _exact_norm(case["post"], s["u"].double(), s["post_gamma"], s["post_beta"])
        out = s["r"].double() * s["res_scale"] + v * s["gate"].double()
        y, m2, r2 = _exact_norm(case["pre"], out, s["pre_gamma"], s["pre_beta"])
        return dict(out=out, stats=torch.stack((m1, r1, m2, r2)), **({} if case["pre"] == "none" else dict(y=y)))
    R, C = case["rows"], case["cols"]
    sums = torch.zeros(5, C, dtype=torch.float64, device="cuda")
    du, dr = (torch.empty(R, C, dtype=torch.float64, device="cuda") for _ in range(2))
    step = max(1, (1 << 25) // C)
    for a in range(0, R, step):  # some rows at a time: the temporaries are large
        at = slice(a, min(a + step, R))
        m1, r1, m2, r2 = s["stats"][:, at].double().unsqueeze(-1)
        g, u = s["dout"][at].double(), s["u"][at].double()
        if case["pre"] != "none":
            dy, z = s["dy"][at].double(), (s["out"][at].double() - m2) * r2
            sums[3] += (dy * z).sum(0)
            sums[4] += dy.sum(0)
            e = dy * s["pre_gamma"].double()
            inner = (e * z).sum(1, keepdim=True) / C
            outer = e.sum(1, keepdim=True) / C if case["pre"] == "layer" else 0.0
            g = g + r2 * (e - outer - z * inner)
        dr[at] = g * s["res_scale"]
        h = g * s["gate"].double()
        if case["post"] == "none":
            sums[2] += (g * u).sum(0)
            du[at] = h
            continue
        z = (u - m1) * r1
        sums[0] += (h * z).sum(0)
        sums[1] += h.sum(0)
        v = z * s["post_gamma"].double() + (s["post_beta"].double() if s["post_beta"] is not None else 0.0)
        sums[2] += (g * v).sum(0)
        e = h * s["post_gamma"].double()
        inner = (e * z).sum(1, keepdim=True) / C
        outer = e.sum(1, keepdim=True) / C if case["post"] == "layer" else 0.0
        du[at] = r1 * (e - outer - z * inner)
    return dict(du=du, dr=dr, dparams=sums)


def _exact_xent(s: dict):
    case = s["case"]
    M, V, K = case["rows"], case["classes"], case["width"]
    w = s["w"].double()
    loss, lse = (torch.zeros(M, dtype=torch.float64, device="cuda") for _ in range(2))
    if case["train"]:
        dx, dw = torch.empty(M, K, dtype=torch.float64, device="cuda"), torch.zeros_like(w)
        dbias = torch.zeros(V, dtype=torch.float64, device="cuda")
    step = max(1, (1 << 28) // V)
    for a in range(0, M, step):  # some rows at a time, with all their classes
        at = slice(a, min(a + step, M))
        x, t = s["x"][at].double(), s["targets"][at]
        l = torch.mm(x, w.t()).mul_(case["scale"])
        if s["bias"] is not None:
            l += s["bias"].double()
        lse[at] = torch.logsumexp(l, 1)
        rows = torch.arange(len(t), device="cuda")[t >= 0]
        picked = t[t >= 0]
        loss[at][rows] = lse[at][rows] - l[rows, picked]
        if not case["train"]:
            continue
        p = l.sub_(lse[at][:, None]).exp_()
        p[rows, picked] -= 1
        p *= (s["grad"][at].double() * (t >= 0))[:, None]
        dx[at] = torch.mm(p, w) * case["scale"]
        dw += torch.mm(p.t().contiguous(), x)
        dbias += p.sum(0)
    if not case["train"]:
        return dict(loss=loss, lse=lse)
    return dict(loss=loss, lse=lse, dx=dx, dw=dw.mul_(case["scale"]), dbias=dbias)


def _exact_clip(s: dict):
    rows = [int(s["count"]) if k == 0 and s["count"] is not None else v.shape[0] for k, v in enumerate(s["grads"])]
    if s["case"]["largest"]:
        norms = torch.tensor([float(v[:n].abs().max()) if n else 0.0 for v, n in zip(s["grads"], rows)], dtype=torch.float64)
        norm = float(norms.max())
    else:
        squares = [float(v[:n].double().square().sum()) for v, n in zip(s["grads"], rows)]
        norms, norm = torch.tensor([math.sqrt(q) for q in squares], dtype=torch.float64), math.sqrt(math.fsum(squares))
    c = s["max_norm"] / norm if norm > s["max_norm"] else 1.0
    out, views = _views(_sizes(s["case"]), dict.fromkeys(TYPES, torch.float64))
    for v, o, n in zip(s["grads"], views, rows):
        o[:n] = v[:n].double() * c
    return dict(norm=torch.tensor([norm], dtype=torch.float64), norms=norms, out=out)


def exact(case: dict, seed: int):
    s = prepare(case, seed)
    return {"xent": _exact_xent, "clip": _exact_clip, "resnorm": _exact_resnorm}[case["kind"]](s)
