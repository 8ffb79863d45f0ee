"""The softmax cross entropy over many classes from its definition in 64 bits, and how far 32-bit sums and the types' roundings may be off.

With u = 2^-24 (half a step of fp32), a logit's sum of n terms is off by at most n u times the sum of magnitudes (n: the width; fp32 operands are
three bfloat16 each, six of whose products are added: n = 6 times the width, and the three products left out are below 2^-24 of a term
together); scale and bias add two roundings.  Powers of two are good to one step (2 u) and their arguments are rounded (u of each magnitude);
sums over classes are added in runs of 16, then by blocks, lanes and tiles.  What a gradient's term d is off by follows from the logit's and lse's
errors, plus its rounding to the type; the products add their own sums' errors, and the result is rounded once.
"""
import torch

U = 2.0 ** -24
HALF_STEP = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.bfloat16, torch.float16)}  # 2^-24, 2^-8, 2^-11; relative, of a normal number
LEAST = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -25}  # half a step of subnormals, and what is flushed


def terms(n, dtype):
    return 6 * n + 4 if dtype is torch.float32 else n + 4


def loss_and_bounds(x, w, targets, bias, scale):
    """lse, loss, their bounds, the logits and theirs"""
    xd, wd = x.double(), w.double()
    l = (xd @ wd.t().contiguous()) * scale
    size = (xd.abs() @ wd.abs().t().contiguous()) * abs(scale)
    if bias is not None:
        l = l + bias.double()
    lse = torch.logsumexp(l, 1) if l.shape[1] else l.new_full((l.shape[0],), -float("inf"))
    have = (targets >= 0) & (targets < l.shape[1])
    at = l.gather(1, targets.clamp(0, max(l.shape[1] - 1, 0))[:, None])[:, 0]
    loss = torch.where(have, lse - at, torch.zeros_like(lse))
    loss = torch.where(have & (lse == -float("inf")), torch.full_like(loss, float("inf")), loss)
    finite = torch.where(torch.isfinite(l), l.abs(), torch.zeros_like(l))
    off = U * (terms(x.shape[1], x.dtype) * size + 6 * finite) + 2.0 ** -120
    tiles = -(-l.shape[1] // 128)
    most = off.amax(1) + U * (120 + tiles + 8 * finite.amax(1))
    return dict(l=l, off=off, lse=lse, loss=loss, lse_off=most, loss_off=2 * most + U * 8 * finite.amax(1), have=have)


def gradients_and_bounds(x, w, targets, bias, scale, grad):
    r = loss_and_bounds(x, w, targets, bias, scale)
    dtype = x.dtype
    live = r["have"] & (grad != 0) & (r["lse"] != -float("inf"))
    g = torch.where(live, grad.double(), torch.zeros_like(r["lse"]))[:, None]
    lse = torch.where(live, r["lse"], torch.zeros_like(r["lse"]))[:, None]
    gap = torch.where(torch.isfinite(r["l"]), (r["l"] - lse).abs(), torch.zeros_like(r["l"]))
    p = torch.where(live[:, None], torch.exp(r["l"] - lse), torch.zeros_like(r["l"]))
    off = p * (r["off"] + r["lse_off"][:, None] + U * (8 + 4 * gap))
    d = p.clone()
    rows = live.nonzero()[:, 0]
    d[rows, targets[rows]] -= 1
    off = (off + U * d.abs()) * g.abs()
    d = d * g
    off = off + 4 * U * d.abs() + 2.0 ** -120  # (grad over the unit, its product, times the unit again)
    dbias = d.sum(0)
    dbias_off = off.sum(0) + U * (x.shape[0] + 4) * d.abs().sum(0) + 2.0 ** -120
    # d as the products take it
    u, least = HALF_STEP[dtype], 0.0
    if dtype is torch.float16:  # held in units of the largest |grad| times 2^14: half a subnormal step is 2^-25
        least = 2.0 ** -25 * 2.0 ** -14 * float(g.abs().max())
    off = off * (1 + u) + u * d.abs() + least
    n = terms(w.shape[0], dtype)
    wd, xd = w.double(), x.double()
    if bias is not None:
        wd = torch.where((bias != -float("inf"))[:, None], wd, torch.zeros_like(wd))
    xd = torch.where(live[:, None], xd, torch.zeros_like(xd))
    dx = (d @ wd) * scale
    dx_off = ((off + U * (n + 4) * d.abs()) @ wd.abs()) * abs(scale)
    dw = (d.t().contiguous() @ xd) * scale
    dw_off = ((off + U * (terms(x.shape[0], dtype) + 4) * d.abs()).t().contiguous() @ xd.abs()) * abs(scale)
    done = lambda v, o: (v, o * (1 + 4 * HALF_STEP[dtype]) + (HALF_STEP[dtype] + 4 * U) * v.abs() + LEAST[dtype] + 2.0 ** -120)  # noqa: E731
    return dict(r, dx=done(dx, dx_off), dw=done(dw, dw_off), dbias=(dbias, dbias_off * (1 + 4 * U)), live=live)


def near(got, want, off, what):
    got, want = got.double(), want.double()
    same = torch.isnan(got) == torch.isnan(want)
    assert bool(same.all()), f"{what}: NaN in {int((~same).sum())} other places"
    infinite = torch.isinf(want) | torch.isinf(got)
    assert bool((got[infinite] == want[infinite]).all()), f"{what}: infinities in other places"
    fine = torch.isfinite(want)
    bad = ((got - want).abs() > off) & fine
    if bool(bad.any()):
        k = int(torch.argmax(torch.where(fine, (got - want).abs() / off, torch.zeros_like(want))))
        raise AssertionError(f"{what}: {int(bad.sum())} of {want.numel()} too far off, worst at {k}: {float(got.flatten()[k])} for "
                             f"{float(want.flatten()[k])}, allowed {float(off.expand_as(want).flatten()[k])}")
