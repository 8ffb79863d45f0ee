"""CPU-only check that the GPU tests' shapes reach every kernel of the layer norm and MXFP4 calls: a change of the rules that choose
between them has to move the shapes too."""
import re

import test_gpu_layernorm as norms
import test_gpu_mxfp4 as products
import test_gpu_mxfp4_kernels as kernels
from launches import FAKE, library_kernels, mx, would_launch

ROOM = 1 << 60
TYPES = (0, 1, 2)


def _launched(calls):
    out = set()
    for rc, launches in would_launch(calls):
        assert rc == 0
        out |= {l.kernel for l in launches}
    return out


def _of_the_library(pattern):
    found = {k for k in library_kernels() if re.match(pattern, k)}
    assert found
    return found


def _product(t, m, n, k):
    return ("dqrm_mxfp4_matmul", mx(m, k), mx(n, k), None, 0, t, FAKE, n, FAKE, ROOM, None)


def test_products_and_linear_layers():
    calls = [_product(t, *s) for t in TYPES for s in kernels.PRODUCTS]
    calls += [("dqrm_mxfp4_linear", t, m, FAKE, k, norm, None, None, 0.0, mx(n, k), None, 0, FAKE, n, FAKE, ROOM, None)
              for t in TYPES for m, n, k in kernels.LINEAR for norm in (0, 1)]
    assert _of_the_library(r"(matmul|matmul_join|few)_kernel") <= _launched(calls)


def test_every_side_of_the_tiles_with_k_whole_and_in_slices():
    seen = {(re.search(r"TileShape<[^>]*>", l[0].kernel).group(0), len(l) > 1)
            for _, l in would_launch([_product(0, *s) for s in kernels.PRODUCTS]) if "TileShape" in l[0].kernel}
    tiles = {re.search(r"TileShape<[^>]*>", k).group(0) for k in _of_the_library("matmul_kernel")}
    assert seen == {(t, sliced) for t in tiles for sliced in (False, True)}


def test_norms():
    shapes = [(t, r, c) for t in TYPES for r, c in norms.SHAPES + [(5000, 40), (2100, 300), (3, 70000)]]
    shapes += [(1 if c % 2 else 2, (1 << 22) // c + 5, c) for c in [100, 250, 384, 500, 1024, 1500, 2048, 2500, 4096, 5001, 8191, 10001, 16384] + kernels.MANY]
    calls = [("dqrm_layernorm_fwd", t, r, c, FAKE, c, None, None, 1e-5, FAKE, c, None, None, None, None) for t, r, c in shapes]
    calls += [("dqrm_layernorm_bwd", t, r, c, FAKE, c, FAKE, c, FAKE, FAKE, None, FAKE, c, FAKE, FAKE, FAKE, ROOM, None) for t, r, c in shapes]
    assert _of_the_library(r"(norm_\w+|join_columns)_kernel") <= _launched(calls)


def test_quantisation():
    calls = []
    for t in TYPES:
        for r, c in products.SHAPES:
            calls += [("dqrm_mxfp4_quant", t, r, c, FAKE, c, None, 0, mx(r, c), by_cols, None, None, 0, None) for by_cols in (None, mx(c, r))]
            calls += [("dqrm_mxfp4_dequant", mx(r, c), t, FAKE, c, None)]
    calls += [("dqrm_mxfp4_quant", 0, 0, 5, FAKE, 5, None, 0, None, None, FAKE, FAKE, ROOM, None)]
    assert _of_the_library(r"(quant_rows|quant_tile|dequant|zero)_kernel") <= _launched(calls)
