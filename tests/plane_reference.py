"""Values of which each plane product counts.  A float is the sum of three bfloat16 planes, and a product of two is taken as six of the nine products
of planes.  In the values here every plane is close to the largest it can be beside the one above it, all of one sign: of a product of two such
values each of the six is at least 2^-17.6, while all that may be wrong with a single product (a sum with nothing else in it) is this, u = 2^-24:
the sums of six exact terms and the scale 7 u, and the three products that are left out 2 2^-8 2^-17 + 2^-34, 1 u."""
import torch

U = 2.0 ** -24
PAIRS = ((0, 0), (0, 1), (1, 0), (1, 1), (0, 2), (2, 0))
PRODUCT = 8 * U  # of a product's magnitude


def values(shape, seed):
    """Floats in [1, 1.25)"""
    g = torch.Generator().manual_seed(seed)
    r = lambda least, most: torch.randint(least, most, shape, generator=g).double()  # noqa: E731
    top = 1 + r(0, 32) * 2.0 ** -7  # 8 bits
    middle = r(250, 256) * 2.0 ** -16  # 8 bits, below half a step of the first plane, 2^-8
    low = r(58, 63) * 2.0 ** -23  # below half a step of the second plane, 2^-17
    v = (top + middle + low).float()
    assert bool((v.double() == top + middle + low).all())
    return v


def planes(v):
    """The three bfloat16 planes, in 64 bits"""
    out, rest = [], v.double()
    for _ in range(3):
        out.append(rest.float().bfloat16().double())
        rest = rest - out[-1]
    return out


def product(a, b, pairs=PAIRS):
    """The products of planes that are asked for, elementwise"""
    a, b = planes(a), planes(b)
    return sum(a[i] * b[j] for i, j in pairs)


def lse_and_bound(logits, exact):
    """lse of a row's logits, and how far one from exact logits may be off: a logit's product and its scale in powers of two, sums over classes (in runs of 16, then
    blocks, lanes and tiles), lse's rounding."""
    lse = torch.logsumexp(exact, 1)
    return torch.logsumexp(logits, 1), (PRODUCT + 2 * U) * exact.abs().amax(1) + U * (120 - (-exact.shape[1] // 128)) + U * lse.abs()
