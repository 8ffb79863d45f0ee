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


def queries(m, v, k, t):
    """What the forward and the backward ask for."""
    (forward, _), (backward, _) = would_launch([("dqrm_softmax_xent_fwd_workspace_bytes", m, v, k, t), ("dqrm_softmax_xent_bwd_workspace_bytes", m, v, k, t)])
    return forward, backward


# long sums in slices: as many rows as a number of tiles has, and one more and less
@pytest.mark.parametrize("t, most, v, k", [(1, 2048, 1024, 2056), (0, 2048, 1000, 1000), (1, 8192, 1024, 2056), (1, 1400, 1024, 8192), (2, 20000, 1024, 8192), (0, 9000, 27, 5541), (0, 3000, 8000, 513),
                                           (1, 130, 1118, 6953), (2, 70, 1000, 4100), (0, 1 << 20, 5, 2080)])
def test_the_workspace_is_enough_for_fewer_rows_whose_sums_go_in_slices(t, most, v, k):
    forward, backward = queries(most, v, k, t)
    rows = {1, 31, 63, 64, 65, 1000, most - 1, most} | {128 * n + e for n in range(1, 66) for e in (-1, 0, 1)}
    rows = sorted(r for r in rows if 1 <= r <= most)
    calls = [(*call[:-2], room, None) for r in rows for call, room in zip(loss(t, r, v, k), (forward, backward))]
    codes = [rc for rc, _ in would_launch(calls)]
    assert set(codes) == {OK}, [(rows[i // 2], "backward" if i % 2 else "forward") for i, rc in enumerate(codes) if rc != OK]


@pytest.mark.parametrize("most, v, k", [(128, 10000, 64), (8192, 200003, 64), (1000, 1_500_000, 8), (5000, 1000, 16), (3000, 130, 64), (40000, 3000, 33), (100, 64, 1)])
def test_the_workspace_is_enough_for_fewer_rows_of_few_columns(most, v, k):
    rows = {1, 2, 33, 64, 65, 127, 128, 129, 191, 192, 193, most // 2, most - 129, most - 128, most - 64, most - 1, most} | {most * n // 40 for n in range(1, 40)}
    rows = sorted(r for r in rows if 1 <= r <= most)
    for t in (0, 1):
        forward, backward = queries(most, v, k, t)
        calls = [(*call[:-2], room, None) for r in rows for call, room in zip(loss(t, r, v, k), (forward, backward))]
        assert {rc for rc, _ in would_launch(calls)} == {OK}, t


def test_the_workspace_of_few_columns_is_what_their_slices_take():
    """dx's and dw's sums are [slices][rows or classes][width] in 32 bits, of as many slices as any plan for so many rows or fewer has."""
    MB = 1 << 20
    # two stages of rows are one slice of dw's sums, 10000 x 64 (2.5 MB); the 157 stages of classes are up to 79 of dx's, 128 x 64 (2.5 MB)
    assert queries(128, 10000, 64, 1)[1] < 8 * MB
    # w's planes 73 MB; 64 tiles of rows, three workgroups to each of 256 CUs: tens of slices of 2 MB of dx's sums, a few of 49 MB of dw's
    assert queries(8192, 200003, 64, 0)[1] < 500 * MB
