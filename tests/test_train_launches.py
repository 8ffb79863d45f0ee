"""CPU-only checks of what the residual norms, the loss and the clip launch, and that the GPU tests' shapes reach every kernel of theirs: a
change of the rules that choose between them has to move the shapes too."""
import re

import pytest

import paper_2410_20046_amd as dq
import test_gpu_residual_norm as norms
import test_gpu_xent as losses
from launches import library_kernels
from train_launches import FAKE, grads, mx, norm, would_launch

OK, ROOM, TYPES = dq.OK, 1 << 60, (0, 1, 2)


def fits(launch):
    return not launch.failed and max(launch.grid[i] * launch.block[i] for i in range(3)) < 1 << 32


def forward(t, rows, cols, q=None):
    return ("dqrm_residual_norm_fwd", t, rows, cols, norm(1, 1), FAKE, cols, FAKE, cols, FAKE, cols, FAKE, cols, FAKE, q, None)


def backward(t, rows, cols):
    return ("dqrm_residual_norm_bwd", t, rows, cols, norm(1, 1), FAKE, cols, FAKE, cols, FAKE, cols, FAKE, cols, FAKE, FAKE, cols, FAKE, cols, FAKE, FAKE, ROOM, None)


def clip(*items):
    return ("dqrm_grad_clip", grads(*items), len(items), 0, 1.0, FAKE, None, FAKE, ROOM, None)


def loss(t, m, v, k):
    return [("dqrm_softmax_xent_fwd", t, m, v, k, FAKE, k, FAKE, k, FAKE, 1.0, FAKE, FAKE, FAKE, FAKE, ROOM, None),
            ("dqrm_softmax_xent_bwd", t, m, v, k, FAKE, k, FAKE, k, FAKE, 1.0, FAKE, FAKE, FAKE, FAKE, k, FAKE, k, FAKE, FAKE, ROOM, None)]


def tensor(k, rows, cols, t=0):
    return (FAKE + (k << 44), rows, cols, cols, None, 0, None, t)


@pytest.mark.parametrize("rows, cols", [((1 << 22) + 5, 40), ((1 << 31) - 2000, 8), (5 << 22, 16384), (1 << 25, 3)])
def test_norms_of_many_rows(rows, cols):
    for t in TYPES:
        for rc, launches in would_launch([forward(t, rows, cols), backward(t, rows, cols)]):
            assert rc == OK and launches and all(map(fits, launches))


@pytest.mark.parametrize("n", [0, 1, 47, 48, 49, 96, 97, 1000])
def test_many_tensors(n):
    """Every tensor's values are in one piece and no other: the pieces follow each other over the launches, in the sums and in the scaling."""
    items = [tensor(k, 1, 1000 * (k % 7) * (k % 11) + (k % 3)) for k in range(n)]
    (rc, launches), = would_launch([clip(*items)])
    assert rc == OK and all(map(fits, launches))
    parts = [l for l in launches if "grad_part" in l.kernel]
    scales = [l for l in launches if "grad_scale" in l.kernel]
    least = 1024 * 8  # values of a piece, as long as there are few
    assert sum(l.grid[0] for l in parts) == sum(-(-i[1] * i[2] // least) for i in items) == sum(l.grid[0] for l in scales)


def test_one_launch_for_each_step_of_a_few_tensors():
    (rc, launches), = would_launch([clip(*[tensor(k, 64, 512) for k in range(13)])])
    assert rc == OK and [re.sub("<.*", "", l.kernel) for l in launches] == ["dqrm_grad::grad_part_kernel", "dqrm_grad::grad_scale_kernel"]


def test_very_large_tensors():
    (rc, launches), = would_launch([clip(tensor(0, 1, 1 << 40), tensor(1, 1 << 30, 1 << 12), tensor(2, 5, 5))])
    assert rc == OK and launches and all(map(fits, launches))


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("m, v, k", [(1, 1 << 30, 64), (64, 1 << 22, 4097), (64, 3, 1 << 22), (65, 1 << 30, 1), (100, (1 << 22) + 5, 33), (1 << 29, 256, 1), (1 << 22, 64, 64),
                                     (129, 1 << 23, 64), (65, 3, 1 << 22), (300, 1 << 20, 100)])
def test_the_loss_of_extreme_shapes(m, v, k, t):
    for rc, launches in would_launch(loss(t, m, v, k)):
        assert rc == OK and launches and all(map(fits, launches))


def of_the_library(name):
    found = {k for k in library_kernels() if name in k}
    assert found
    return found


def launched(calls):
    out = set()
    for rc, made in would_launch(calls):
        assert rc == OK
        out |= {l.kernel for l in made}
    return out


def test_the_norms_kernels_are_tested():
    calls = []
    for t in TYPES:
        for r, c in norms.SHAPES + norms.MANY:
            calls += [forward(t, r, c, mx(r, c)), forward(t, r, c), backward(t, r, c)]
    missing = of_the_library("dqrm_resnorm") - launched(calls)
    assert not missing, missing


def test_the_losses_kernels_are_tested():
    calls = []
    shapes = [(t, *s) for t in TYPES for s in losses.SHAPES + [(m, 70001, 17) for m in (1, 2, 3, 4, 5, 8, 9, 16)]] + [
        ({"f32": 0, "bf16": 1, "f16": 2}[t], *s) for t, *s in losses.PIECES]
    for shape in shapes:
        calls += loss(*shape)
    missing = (of_the_library("xent")) - launched(calls)
    assert not missing, missing


def test_the_clips_kernels_are_tested():
    calls = [("dqrm_grad_clip", grads(tensor(0, 5, 5)), 1, kind, 1.0, FAKE, None, FAKE, ROOM, None) for kind in (0, 1)]
    calls += [("dqrm_grad_norm", grads(tensor(0, 5, 5)), 1, kind, FAKE, None, FAKE, ROOM, None) for kind in (0, 1)]
    missing = of_the_library("dqrm_grad") - launched(calls)
    assert not missing, missing
