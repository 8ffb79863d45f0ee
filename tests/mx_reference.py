"""Plain references of MXFP4 and of layer norm in 64 bits (numpy), written from the definitions, for the tests of the kernels."""
import numpy as np
import torch

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
#: half a unit in the last place of each type, relative
HALF_ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
ULP = HALF_ULP["f32"]
#: the smallest subnormal of each type: values below the normal range are off by half of it at most
TINY = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -24}


def pad128(n):
    return -(-n // 128) * 128


def quantise(x):
    """(magnitude index and sign as a code [R][P], scale bytes [R][P / 32]) of x [R][C] in 64 bits, P = C padded to 128."""
    R, C = x.shape
    v = np.zeros((R, pad128(C)))
    v[:, :C] = x
    v = v.reshape(R, -1, 32)
    bad = ~np.isfinite(v).all(-1)
    amax = np.where(bad, 1.0, np.abs(np.where(np.isfinite(v), v, 0)).max(-1))
    _, e = np.frexp(amax)  # amax = f 2^e, 1/2 <= f < 1
    e = np.maximum(np.where(amax > 0, e - 1 - 2, -127), -127)
    m = np.ldexp(np.abs(np.where(np.isfinite(v), v, 0)), -e[..., None])
    d = np.abs(m[..., None] - MAGNITUDES)
    near = d.min(-1, keepdims=True)
    hit = d == near  # one code, or the two that a midpoint lies between: of those the even one
    even = hit & (np.arange(8) % 2 == 0)
    code = np.where(hit.sum(-1) == 1, hit.argmax(-1), even.argmax(-1))
    code = code | (np.signbit(v).astype(np.int64) << 3)
    code[bad] = 0
    scale = np.where(bad, 255, e + 127)
    scale[~bad & (amax == 0)] = 0
    return code.reshape(R, -1).astype(np.uint8), scale.astype(np.uint8)


def pack(code):
    return (code[:, 0::2] | (code[:, 1::2] << 4)).astype(np.uint8)


def values(codes, scales, cols):
    """What packed codes and scale bytes stand for, in 64 bits."""
    code = np.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[0], -1)
    v = np.where(code & 8, -1.0, 1.0) * MAGNITUDES[code & 7]
    s = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    return (v * np.repeat(s, 32, 1))[:, :cols]


def quantised_values(x):
    c, s = quantise(x)
    return values(pack(c), s, x.shape[1])


def norm(x, gamma, beta, eps):
    mean = x.mean(1)
    d = x - mean[:, None]
    rstd = 1.0 / np.sqrt((d * d).mean(1) + eps)
    return d * rstd[:, None] * gamma + beta, mean, rstd


def norm_backward(dy, x, mean, rstd, gamma):
    xh = (x - mean[:, None]) * rstd[:, None]
    g = dy * gamma
    dx = rstd[:, None] * (g - g.mean(1, keepdims=True) - xh * (g * xh).mean(1, keepdims=True))
    return dx, (dy * xh).sum(0), dy.sum(0)


def on_gpu(a, dtype, stride=None, offset=0):
    """`a` as a matrix of `dtype` on the GPU with the given row stride, its first element `offset` elements into its memory;
    everything around it is NaN."""
    a = torch.as_tensor(np.ascontiguousarray(a)).to(dtype)
    R, C = a.shape
    stride = C if stride is None else stride
    room = torch.full((offset + R * stride + 16,), float("nan"), dtype=dtype, device="cuda")
    view = room[offset:offset + R * stride].view(R, stride)[:, :C]
    view.copy_(a)
    return view


def f64(t):
    return t.detach().cpu().double().numpy()


def sum_steps(n):
    """Roundings that a value goes through in a row's sum, at most: 32 values to a thread in turn (longer rows: one chunk of 8
    after another by each of 256 threads), then a tree."""
    return 40 + n / 2048


def backward_bounds(dy, x, mean, rstd, gamma, dx, dtype, chain):
    n = x.shape[1]
    s = sum_steps(n) + 6
    xh = np.abs((x - mean[:, None]) * rstd[:, None])
    # (x - mean) rstd: two roundings
    g = np.abs(dy * gamma)
    b_dx = rstd[:, None] * (3 * ULP * g + s * ULP * g.mean(1, keepdims=True) + (s + 6) * ULP * xh * (g * xh).mean(1, keepdims=True)) + 3 * ULP * np.abs(dx)
    return (2 * b_dx + 1.01 * HALF_ULP[dtype] * np.abs(dx) + TINY[dtype], 1.01 * (chain + 3) * ULP * (np.abs(dy) * xh).sum(0) + 1e-45,
            1.01 * chain * ULP * np.abs(dy).sum(0) + 1e-45)
