"""CPU-only checks of what the layer norm and MXFP4 calls launch: the host side runs with the HIP runtime's launch calls written down
instead of made (see launches.py)."""
import random

import pytest

import paper_2410_20046_amd as dq
from launches import FAKE, mx, would_launch

OK, INVALID, UNSUPPORTED = dq.OK, dq.ERR_INVALID_ARG, dq.ERR_UNSUPPORTED
BF16 = dq.BF16
ROOM = 1 << 60  # bytes of workspace: enough for anything


def threads(launch):
    return max(launch.grid[i] * launch.block[i] for i in range(3))


def norm_fwd(rows, cols):
    return ("dqrm_layernorm_fwd", BF16, rows, cols, FAKE, cols, None, None, 1e-5, FAKE, cols, None, None, None, None)


def norm_bwd(rows, cols, dx=FAKE, sums=FAKE):
    return ("dqrm_layernorm_bwd", BF16, rows, cols, FAKE, cols, FAKE, cols, FAKE, FAKE, None, dx, cols, sums, sums, FAKE, ROOM, None)


@pytest.mark.parametrize("call", [norm_fwd, norm_bwd])
@pytest.mark.parametrize("rows, cols, block", [((1 << 22) - 1, 16385, 1024), (1 << 22, 16385, 1024), ((1 << 22) + 1, 40000, 1024), (5 << 22, 16385, 1024),
                                               (1 << 25, 3, 64), ((1 << 25) + 1, 7, 64)])
def test_norms_of_many_rows_that_are_read_more_than_once(call, rows, cols, block):
    """A workgroup to a row, of 1024 threads where rows are long: a launch has fewer than 2^32 threads, and all launches every row."""
    (rc, launches), = would_launch([call(rows, cols)])
    assert rc == OK
    assert all(threads(l) < 1 << 32 and not l.failed for l in launches)
    long = [l for l in launches if "_long_kernel" in l.kernel]
    assert all(l.block[0] == block for l in long) and sum(l.grid[0] for l in long) == rows


def quant(rows, cols, by_rows=None, by_cols=None, sums=None):
    return ("dqrm_mxfp4_quant", BF16, rows, cols, FAKE, cols, None, 0, by_rows, by_cols, sums, FAKE, ROOM, None)


@pytest.mark.parametrize("cols", [1, 8190, (1 << 28) - 16, (1 << 28) - 15, 1 << 28, (1 << 29) + 17])
@pytest.mark.parametrize("pair", [False, True])
def test_column_sums_of_very_wide_matrices(cols, pair):
    """The join of partial sums has 16 threads to a column, one pair of arrays of sums or one array, and is as many launches as it takes."""
    (rc, launches), = would_launch([norm_bwd(129, cols, dx=None) if pair else quant(129, cols, sums=FAKE)])
    if not pair and 2 * -(-cols // 128) > 1 << 23:  # more tiles of 128 by 128 than the quantisation takes
        assert rc == UNSUPPORTED and not launches
        return
    assert rc == OK
    assert all(threads(l) < 1 << 32 and not l.failed for l in launches)
    joins = [l for l in launches if l.kernel == "join_columns_kernel"]
    assert all(l.grid[1] == (2 if pair else 1) for l in joins)
    assert sum(l.grid[0] for l in joins) == -(-cols // 16)


def linear(m, n, k, norm=0, ws_bytes=ROOM):
    return ("dqrm_mxfp4_linear", BF16, m, FAKE, k, norm, None, None, 1e-5, mx(n, k), None, 0, FAKE, n, FAKE, ws_bytes, None)


def matmul(m, n, k, ws_bytes=ROOM):
    return ("dqrm_mxfp4_matmul", mx(m, k), mx(n, k), None, 0, BF16, FAKE, n, FAKE, ws_bytes, None)


@pytest.mark.parametrize("m, n, k", [(1 << 20, 1 << 19, 64), (1 << 30, 1000, 300), (1 << 27, 8193, 17), (1 << 20, 1 << 18, (1 << 24) + 1)])
def test_products_that_are_refused_launch_nothing(m, n, k):
    """More outputs than 2^22 tiles of 256 by 256 hold, and longer sums than 2^24: the linear layer's activations stay unquantised too."""
    for rc, launches in would_launch([matmul(m, n, k), linear(m, n, k), linear(m, n, k, norm=1)]):
        assert rc == UNSUPPORTED and not launches


def test_products_up_to_the_limit_are_launched():
    for rc, launches in would_launch([f(*shape) for shape in ((1 << 20, 1 << 18, 64), (64, (1 << 30) + 5, 1100), (3, (1 << 30) + 5, 64))
                                      for f in (matmul, linear, lambda *s: linear(*s, norm=1))]):
        assert rc == OK and launches and all(threads(l) < 1 << 32 and not l.failed for l in launches)


def held(what, *shape):
    return ("dqrm_" + what + "_workspace_bytes", *shape)


def fewer(m, rng):
    """Numbers of rows up to m: the smallest, those around each multiple of a tile's rows that a plan changes at, and others."""
    near = {1, 2, 16, 17, 32, 33, 64, 65, 127, 128, 129, 255, 256, 257, 512, 513, 1024, 2048, 4096, m - 1, m, m // 2, m // 3}
    return sorted(v for v in near | {rng.randint(1, m) for _ in range(30)} if 1 <= v <= m)


@pytest.mark.parametrize("n, k", [(512, 8192), (2048, 16384), (1, 65536), (367, 65536), (130, 33000), (1000, 60001), (8192, 8192), (4100, 4099), (77, 40000)])
@pytest.mark.parametrize("m", [64, 1000, 8192, 20000])
def test_the_workspace_of_a_product_is_enough_for_fewer_rows(m, n, k):
    """One workspace for the largest batch serves smaller ones, the last batch of an epoch and single requests among them."""
    some = fewer(m, random.Random(m + n + k))
    (product, _), (layer, _) = would_launch([held("mxfp4_matmul", m, n, k), held("mxfp4_linear", m, n, k)])
    for call, room in ((matmul, product), (linear, layer)):
        assert [rc for rc, _ in would_launch([call(v, n, k, ws_bytes=room) for v in some])] == [OK] * len(some)


@pytest.mark.parametrize("cols", [1, 7, 40, 300, 1200, 4100, 8192, 16384, 16385, 50000])
@pytest.mark.parametrize("rows", [3, 65, 1000, 4097, 100000])
def test_the_other_workspaces_are_enough_for_fewer_rows(rows, cols):
    some = fewer(rows, random.Random(rows + cols))
    (norm, _), (sums, _) = would_launch([held("layernorm_bwd", rows, cols), held("mxfp4_quant", rows, cols)])
    back = [("dqrm_layernorm_bwd", t, v, cols, FAKE, cols, FAKE, cols, FAKE, FAKE, None, FAKE, cols, FAKE, FAKE, FAKE, norm, None) for v in some for t in (0, 1, 2)]
    quantised = [("dqrm_mxfp4_quant", 0, v, cols, FAKE, cols, None, 0, None, None, FAKE, FAKE, sums, None) for v in some]
    assert {rc for rc, _ in would_launch(back + quantised)} == {OK}
