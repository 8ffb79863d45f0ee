"""Gradients that are not scaled: what `out` gets is a copy, bit for bit."""
import math

import pytest
import torch

import paper_2410_20046_amd as dq
from test_gpu_grad_clip import TYPES, space

pytestmark = pytest.mark.gpu

# quiet and signalling NaNs with and without payload, infinities, subnormals, zeros of both signs
BITS = {"f32": (torch.int32, [0x7FC00000, 0x7F800001, 0x7FABCDEF, -0x7FFFFF, -1, 0x7F800000, -0x800000, 1, 0x7FFFFF, -0x80000000, 0, 0x3F800000]),
        "bf16": (torch.int16, [0x7FC0, 0x7F81, 0x7FAB, -0x7F, -1, 0x7F80, -0x80, 1, 0x7F, -0x8000, 0, 0x3F80]),
        "f16": (torch.int16, [0x7E00, 0x7C01, 0x7DAB, -0x3FF, -1, 0x7C00, -0x400, 1, 0x3FF, -0x8000, 0, 0x3C00])}


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(5000,), (100, 13), (300, 3), (7, 8)])
def test_a_copy_has_the_same_bits(dtype, shape):
    whole, patterns = BITS[dtype]
    n = math.prod(shape)
    bits = torch.tensor(patterns, device="cuda").repeat(n // len(patterns) + 1)[:n].to(whole).view(shape)
    t, place = bits.view(TYPES[dtype]), torch.zeros(shape, dtype=TYPES[dtype], device="cuda")
    if len(shape) == 2:  # rows with gaps
        place = torch.zeros(shape[0], shape[1] + 3, dtype=TYPES[dtype], device="cuda")[:, 1:-2]
    grads = dq.Grads([t], out=[place])
    norm = torch.empty(1, device="cuda")
    dq.dqrm_grad_clip(grads, 0.5, norm, workspace=space(grads))
    assert math.isnan(float(norm)) and torch.equal(place.contiguous().view(whole), bits)
    for given in (math.nan, math.inf, 0.25):
        place.zero_()
        dq.dqrm_grad_scale(grads, torch.tensor([given], device="cuda"), 0.5)
        assert torch.equal(place.contiguous().view(whole), bits), given
