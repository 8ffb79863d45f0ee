"""CPU-only checks of what the loss launches at the limits of its sizes, and of what it asks of its workspace."""
import pytest

import paper_2410_20046_amd as dq
from test_train_launches import fits, loss
from train_launches import would_launch

OK = dq.OK


@pytest.mark.parametrize("t", (0, 1, 2))
@pytest.mark.parametrize("m, v, k", [(1 << 19, 1 << 19, 128), (1 << 19, 1 << 19, 100), (1 << 18, 1 << 20, 128), (1 << 30, 256, 65), (1 << 30, 256, 70), (1 << 30, 200, 100),
                                     (1 << 30, 256, 256), (1 << 29, 500, 100), (1 << 29, 512, 512), ((1 << 30) - 5, 129, 200), (1 << 20, 1 << 18, 512)])
def test_short_sums_of_many_tiles(m, v, k, t):
    """Sums of few stages take small tiles, and the largest sizes are counted in large ones: no launch has 2^32 threads."""
    for rc, launches in would_launch(loss(t, m, v, k)):
        assert rc == OK and launches and all(map(fits, launches))
