"""The example that runs the operators together: it learns, and its requests agree with its batches."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_click_model_learns_and_serves(dtype):
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import mxfp4_top_mlp
    finally:
        sys.path.pop(0)
    first, last, worst = mxfp4_top_mlp.run(steps=120, batch=1000, hidden=(200, 72), dtype=dtype, say=lambda *a: print(*a, flush=True))
    # labels are a coin's at the start (ln 2); a model that learns nothing stays there
    assert last < 0.75 * first and last < 0.6
    # a batch's and a request's norms add in other orders: single values may take the neighbouring 4-bit code, here and there
    assert worst < 0.02


@pytest.mark.parametrize("batch", [1, 3])
def test_click_model_of_few_samples(batch):
    """Batches smaller than the requests that the example ends with."""
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import mxfp4_top_mlp
    finally:
        sys.path.pop(0)
    first, last, worst = mxfp4_top_mlp.run(steps=2, batch=batch, hidden=(40,), say=lambda *a: print(*a, flush=True))
    # (a code that a request's norm takes the other side of moves a layer of 40 outputs by more than a tolerance of use)
    assert all(abs(v) < float("inf") for v in (first, last, worst))
