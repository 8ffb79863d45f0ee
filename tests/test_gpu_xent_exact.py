"""The loss where its logits are known exactly, so that nothing but what follows them counts.

With u = 2^-24: a logit in powers of two is rounded to u of itself and more than that a constant's rounding, which is the same for all of a row; so the
maximum and a term beside it are off by 2.1 u of the logit together, a term's power by as much of itself, and the sum (of the maximum's 1 and a
few terms, in runs) by its rounding.  The loss is (maximum - target's logit) + log of the sum: exact but for that where the target is the maximum."""
import pytest
import torch

from test_gpu_xent import backward, forward

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF = {t: torch.finfo(t).eps / 2 for t in TYPES.values()}

# of each kernel: a few rows, strips, tiles of few rows, widths up to 64, tiles, the largest tiles, sums in slices
KERNELS = [("f32", 1, 300, 40), ("f32", 4, 300, 40), ("f32", 60, 300, 40), ("f32", 130, 300, 40), ("f32", 130, 300, 72), ("f32", 130, 300, 1100), ("f32", 1030, 33000, 104)] + [
    (t, *s) for t in ("bf16", "f16") for s in ((60, 300, 41), (60, 300, 40), (130, 300, 40), (130, 300, 136), (1030, 33000, 600), (130, 300, 2056))]

# a, g: logits of a, a - g and (all other classes) a - 8 g, exact in each type
PAIRS = [(1000, 10), (1000, 12), (992, 9), (720, 10), (600, 10), (2000, 9), (4000, 7), (-1000, 9), (250, 12), (0, 16), (512, 11), (-720, 10)]


def known(m, v, k, dtype):
    """x, w, the rows' a and g.  Beside the two columns of the logits two that x has zeros in: of class 0, and of class 1."""
    t = TYPES[dtype]
    a, g = (torch.tensor([p[i] for p in PAIRS], dtype=torch.float64, device="cuda").repeat(m // len(PAIRS) + 1)[:m] for i in (0, 1))
    x, w = torch.zeros(m, k, dtype=t, device="cuda"), torch.zeros(v, k, dtype=t, device="cuda")
    x[:, 3], x[:, k - 2] = a.to(t), g.to(t)
    w[:, 3], w[:, k - 2] = 1, -8
    w[0, k - 2], w[1, k - 2] = 0, -1
    w[0, 5], w[1, k - 5] = 1, 1
    return x, w, a, g


@pytest.mark.parametrize("dtype, m, v, k", KERNELS)
def test_a_loss_near_zero_of_large_logits(dtype, m, v, k):
    x, w, a, g = known(m, v, k, dtype)
    beside = torch.exp(-g) + (v - 2) * torch.exp(-8 * g)
    least = U * (2.1 * a.abs() + 2.1 * 8 * g + 8)  # of a term
    for target in (0, 1):
        loss, lse = forward(x, w, torch.full((m,), target, device="cuda"))
        want = torch.log1p(beside) + target * g
        off = beside * least + 8 * U + target * U * 2.1 * a.abs() + 2 * U * want
        assert bool(((loss.double() - want).abs() <= off).all()), float(((loss.double() - want).abs() / off).max())
        want = a + torch.log1p(beside)
        # the maximum's rounding, the constant's, that of lse
        off = beside * least + 8 * U + 2.4 * U * a.abs()
        assert bool(((lse.double() - want).abs() <= off).all()), float(((lse.double() - want).abs() / off).max())


@pytest.mark.parametrize("dtype, m, v, k", KERNELS)
def test_gradients_are_off_by_no_more_than_lse_is_rounded(dtype, m, v, k):
    """exp(l - lse) has lse's rounding to 32 bits, half a step of it, and beside it a few roundings of numbers around 1; dx of the columns that are one class's
    alone is that class's d, rounded to the type twice."""
    x, w, a, g = known(m, v, k, dtype)
    targets = torch.zeros(m, dtype=torch.int64, device="cuda")
    _, lse = forward(x, w, targets)
    dx, _, _ = backward(x, w, targets, lse, torch.ones(m, device="cuda"))
    total = 1 + torch.exp(-g) + (v - 2) * torch.exp(-8 * g)
    half = torch.exp2(torch.floor(torch.log2(lse.double().abs().clamp(min=2.0 ** -20))) - 24)
    step = HALF[TYPES[dtype]] * (0 if dtype == "f32" else 2.1)
    for column, want, more in ((5, 1 / total - 1, 0.0), (k - 5, torch.exp(-g) / total, 2.1 * U * a.abs())):
        off = (1 if column == 5 else want) * (1.02 * half + more + 10 * U) + step * want.abs() + (2.0 ** -24 if dtype == "f16" else 0.0)
        got = dx[:, column].double()
        assert bool(((got - want).abs() <= off).all()), (column, float(((got - want).abs() / off).max()))


@pytest.mark.parametrize("dtype, m, v, k", [s for s in KERNELS if s[0] == "f16"])
def test_the_range_of_gradients_in_half(dtype, m, v, k):
    """d is held in units of the largest |grad| times 2^14: a d of that size has fp16's bits down to 2^-28 of it, half a step of the subnormals is 2^-39 of it, and
    what is below that is zero.  Class 0 has all the weight and class 1 is the target: d of class 0, which is dx's column of its own, is grad."""
    x, w, a, g = known(m, v, k, dtype)
    below = torch.arange(m, device="cuda", dtype=torch.float64) % 46
    grad = torch.exp2(15 - below)
    targets = torch.ones(m, dtype=torch.int64, device="cuda")
    _, lse = forward(x, w, targets)
    dx, _, _ = backward(x, w, targets, lse, grad.float())
    want, got = grad / (1 + torch.exp(-g) + (v - 2) * torch.exp(-8 * g)), dx[:, 5].double()
    step = want * (2.1 * HALF[torch.float16] + 2.0 ** -24 * (a.abs() + 10)) + 2.0 ** -25  # d's rounding and the result's, lse's; the result's subnormals
    assert bool(((got - want).abs() <= step)[below <= 28].all()) and bool((want[below <= 28] >= 2.0 ** -14).all())
    assert bool(((got - want).abs() <= step + 2.0 ** (15 - 39)).all())
    assert bool((dx[below >= 40] == 0).all()) and bool((got[below < 38] > 0).all())
