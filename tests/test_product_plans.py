"""How feed-forward products are cut (host arithmetic), and that the tests of the tiles leave none of them out."""

import ctypes
import os

import pytest

import ff_common as F
from paper_2002_09481_amd import binding as ax
from test_gpu_matmul_tiles import CASES

pytestmark = pytest.mark.skipif(not os.path.exists(ax.LIB_PATH), reason="libaxconv.so not built")


def test_every_tile_is_among_the_cases():
    """Of each product: all tiles that some size takes, in one piece and in slices."""
    seen = {}
    for product, dt, transposed, M, K, N, rows, sliced in CASES:
        plan = ax.ax_probe_product_plan(product, M, K, N, F.DT[dt], None, transposed)
        assert plan["kernel"] == "tiles" and plan["tile"][0] == rows and (plan["slices"] > 1) == sliced, plan
        seen.setdefault((product, dt, transposed), set()).add((rows, sliced))
    assert len(seen) == 20  # products x types x layouts
    for (product, dt, transposed), have in seen.items():
        for M in (33, 257, 1531, 4096, 8192):
            for K in (64, 1000, 4096, 8192):
                for N in (64, 1000, 4096, 16384):
                    plan = ax.ax_probe_product_plan(product, M, K, N, F.DT[dt], None, transposed)
                    if plan["kernel"] == "tiles":
                        assert (plan["tile"][0], plan["slices"] > 1) in have, (product, dt, transposed, M, K, N, plan)


def test_few_rows():
    plan = ax.ax_probe_product_plan
    assert plan("matmul", 1, 4096, 4096) == {"kernel": "few", "tile": (0, 0), "slices": 1}
    assert plan("matmul", 16, 8192, 512, F.DT["f32"])["slices"] > 1
    assert plan("matmul_gx", 8, 512, 512, F.DT["f32"])["kernel"] == "few" and plan("matmul_gw", 8, 512, 512, F.DT["f32"])["kernel"] == "outer"
    assert plan("matmul", 0, 64, 64)["slices"] == 1


def test_refusals():
    L, d = ax.lib(), ax.ax_matmul_desc_t(4, 64, 32, 32, 64, 64, 64, 1, 1, 0, 0, 0)
    R, none = ctypes.byref, [None] * 4
    assert L.ax_probe_product_plan(R(d), 0, *none) == 0
    assert L.ax_probe_product_plan(None, 0, *none) == -1
    for product in (-1, 8, 1, 3):  # codes are [N, K]
        assert L.ax_probe_product_plan(R(d), product, *none) == -8
    d.N = 0
    assert L.ax_probe_product_plan(R(d), 0, *none) == -2
