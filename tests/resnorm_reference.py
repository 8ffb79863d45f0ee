"""Residual joins with their norms in 64 bits, and how far 32-bit arithmetic may be off: each step's rounding (u = 2^-24 of its result) and what
the errors of its operands make of it, to first order; twice that is allowed, and one rounding to the type (half a step)."""
import torch

from mx_reference import HALF_ULP, TINY, sum_steps

U = 2.0 ** -24
NAMES = {torch.float32: "f32", torch.bfloat16: "bf16", torch.float16: "f16"}


def rounded(v, off, dtype):
    name = NAMES[dtype]
    return 2 * off + 1.01 * HALF_ULP[name] * v.abs() + TINY[name]


def norm(kind, v, off, gamma, beta, eps):
    """(normalised with gain and offset, its bound, mean, rstd, their bounds); kind: none, layer, rms"""
    if kind == "none":
        return v, off, None, None, None, None
    s = sum_steps(v.shape[1])
    mean, off_mean = torch.zeros_like(v[:, :1]), torch.zeros_like(v[:, :1])
    if kind == "layer":
        mean, off_mean = v.mean(1, keepdim=True), (s + 2) * U * v.abs().mean(1, keepdim=True) + off.mean(1, keepdim=True)
    d = v - mean
    off_d = off + off_mean + U * d.abs()
    off_var = (2 * d.abs() * off_d).mean(1, keepdim=True) + off_d.amax(1, keepdim=True) ** 2 + (s + 4) * U * (d * d).mean(1, keepdim=True)
    rstd = ((d * d).mean(1, keepdim=True) + eps) ** -0.5
    off_rstd = 0.5 * off_var * rstd ** 3 + 4 * U * rstd
    z = d * rstd
    off_z = off_d * rstd + d.abs() * off_rstd + U * z.abs()
    y = z * gamma + beta
    return y, off_z * gamma.abs() + 3 * U * (z * gamma).abs() + U * (beta.abs() + y.abs()), mean, rstd, off_mean, off_rstd


def forward(p, u, r):
    """p: dict(post, pre, post_gamma, post_beta, gate, pre_gamma, pre_beta (64-bit, ones and zeros for None), res_scale, eps)"""
    zero = torch.zeros_like(u)
    v, off_v, m1, r1, b_m1, b_r1 = norm(p["post"], u, zero, p["post_gamma"], p["post_beta"], p["eps"])
    out = p["res_scale"] * r + p["gate"] * v
    off_out = p["gate"].abs() * (off_v + 4 * U * (v.abs() + p["post_beta"].abs())) + 2 * U * ((p["res_scale"] * r).abs() + out.abs())
    y, off_y, m2, r2, b_m2, b_r2 = norm(p["pre"], out, off_out, p["pre_gamma"], p["pre_beta"], p["eps"])
    return dict(out=(out, off_out), y=(y, off_y), stats=[(m1, b_m1), (r1, b_r1), (m2, b_m2), (r2, b_r2)])


def backward_norm(kind, e, off_e, z, rstd):
    """rstd (e - mean(e) - z mean(e z)) and its bound; e: the gradient times the gain"""
    s = sum_steps(z.shape[1])
    mean = lambda v: v.mean(1, keepdim=True)  # noqa: E731
    c0, off_c0 = (mean(e), mean(off_e) + (s + 2) * U * mean(e.abs())) if kind == "layer" else (0.0, 0.0)
    c1 = mean(e * z)
    off_c1 = mean(off_e * z.abs()) + (s + 5) * U * mean((e * z).abs())
    v = rstd * (e - c0 - z * c1)
    return v, rstd * (off_e + off_c0 + z.abs() * off_c1 + 5 * U * (z * c1).abs() + 3 * U * e.abs()) + 4 * U * v.abs()


def backward(p, dout, dy, u, out, stats):
    """stats: the forward's, [4][rows] in 64 bits"""
    m1, r1, m2, r2 = (s[:, None] for s in stats)
    g, off_g = dout, torch.zeros_like(dout)
    n, rows = dout.shape[1], dout.shape[0]
    chain = rows / 256 + 80  # a thread's rows, a workgroup's groups of rows, its lanes' and their join
    columns = lambda t, off=0.0: (t.sum(0), 2 * (off + (chain + 4) * U * t.abs()).sum(0) + 1e-37)  # noqa: E731
    zero = torch.zeros(n, dtype=torch.float64, device=dout.device)
    pre_gamma = pre_beta = post_gamma = post_beta = (zero, zero)
    if p["pre"] != "none":
        z2 = (out - m2) * r2
        pre_gamma, pre_beta = columns(dy * z2, 3 * U * (dy * z2).abs()), columns(dy)
        e = dy * p["pre_gamma"]
        d, off_d = backward_norm(p["pre"], e, U * e.abs(), z2, r2)
        g = g + d
        off_g = off_d + U * g.abs()
    z1 = (u - m1) * r1 if p["post"] != "none" else u
    s0, off_s0 = columns(g, off_g)
    s1, off_s1 = columns(g * z1, off_g * z1.abs() + 3 * U * (g * z1).abs())
    h = g * p["gate"]
    off_h = off_g * p["gate"].abs() + U * h.abs()
    du, off_du = h, off_h
    gate = (s1, off_s1)
    if p["post"] != "none":
        e = h * p["post_gamma"]
        du, off_du = backward_norm(p["post"], e, off_h * p["post_gamma"].abs() + U * e.abs(), z1, r1)
        post_gamma, post_beta = ((p["gate"] * s, p["gate"].abs() * off + 2 * U * (p["gate"] * s).abs()) for s, off in ((s1, off_s1), (s0, off_s0)))
        total = p["post_gamma"] * s1 + p["post_beta"] * s0
        gate = total, p["post_gamma"].abs() * off_s1 + p["post_beta"].abs() * off_s0 + 4 * U * ((p["post_gamma"] * s1).abs() + (p["post_beta"] * s0).abs())
    dr = p["res_scale"] * g
    return dict(du=(du, off_du), dr=(dr, abs(p["res_scale"]) * off_g + U * dr.abs()), dparams=[post_gamma, post_beta, gate, pre_gamma, pre_beta])
