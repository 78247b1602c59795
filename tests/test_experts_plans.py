"""How products grouped by expert and products with 4-bit weights are cut (host arithmetic), and that the tests of their kernels leave
none of them out."""

import ctypes
import os

import pytest

import ff_common as F
from paper_2002_09481_amd import binding as ax
from test_gpu_experts_tiles import CASES, Q4_CASES

pytestmark = pytest.mark.skipif(not os.path.exists(ax.LIB_PATH), reason="libaxconv.so not built")


def test_every_tile_is_among_the_cases():
    seen = {}
    for product, dt, transposed, found, rows, E, K, N, high, per_cu in CASES:
        plan = ax.ax_probe_experts_plan(product, rows, E, K, N, F.DT[dt], transposed, x_rows=rows // 2 + 1 if found else None)
        assert (plan["kernel"], plan["tile"][0], plan["per_cu"], plan["found"]) == ("tiles", high, per_cu, found), (plan, product, rows, E, K, N)
        seen.setdefault((product, dt, transposed, found), set()).add((high, per_cu))
    assert len(seen) == 21  # products x types x layouts x rows in order or looked up
    for (product, dt, transposed, found), have in seen.items():
        for rows in (33, 257, 2051, 16411):
            for E in (1, 5, 33):
                for K in (40, 1000, 4104):
                    for N in (40, 1000, 4100):
                        plan = ax.ax_probe_experts_plan(product, rows, E, K, N, F.DT[dt], transposed, x_rows=rows // 2 + 1 if found else None)
                        if plan["kernel"] == "tiles":
                            assert (plan["tile"][0], plan["per_cu"]) in have, (product, dt, transposed, found, rows, E, K, N, plan)


def test_every_kernel_of_4_bit_products_is_among_the_cases():
    seen = {}
    for gated, dt, rows, E, K, N, kernel, high, cols, waves in Q4_CASES:
        plan = ax.ax_probe_q4_plan(gated, rows, E, K, N, 64, F.DT[dt])
        assert (plan["kernel"], plan["tile"], plan["waves"]) == (kernel, (high, cols), waves), (plan, gated, dt, rows, E, K, N)
        seen.setdefault((gated, dt), set()).add((kernel, high, cols, waves))
    assert len(seen) == 4
    for (gated, dt), have in seen.items():
        for rows in (1, 17, 33, 130, 700, 4100):
            for E in (1, 5, 33):
                for K in (40, 1000, 4104):
                    for N in (40, 264, 1000, 4100, 8200):
                        plan = ax.ax_probe_q4_plan(gated, rows, E, K, N, 64, F.DT[dt])
                        assert (plan["kernel"], *plan["tile"], plan["waves"]) in have, (gated, dt, rows, E, K, N, plan)


def test_few_rows_and_rows_that_are_copied():
    plan = ax.ax_probe_experts_plan
    assert plan("matmul", 8, 8, 1000, 1000)["kernel"] == "few" and plan("matmul", 0, 8, 1000, 1000)["tile"] == (0, 0)
    assert plan("gated", 4000, 2, 1000, 1000, x_rows=3000)["found"] and not plan("gated", 4000, 2, 1001, 1000, x_rows=3000)["found"]
    assert not plan("gated", 4000, 2, 1000, 1000, x_rows=3000, unaligned=True)["found"]
    assert not plan("gated", 4000, 2, 1000, 1000, F.DT["f32"], x_rows=3000)["found"]
    assert not plan("gated", 4000, 2, 8192, 64, x_rows=1 << 17)["found"]  # 2 GB of x: copied


def test_an_empty_x_is_not_read():
    """Rows of an x that has none, all of zeros: only the copies know what to do with those."""
    for rows, dt in ((4, "bf16"), (4, "f32"), (4000, "bf16"), (4000, "f32")):
        plan = ax.ax_probe_experts_plan("matmul", rows, 2, 1000, 1000, F.DT[dt], x_rows=0)
        assert plan["kernel"] == "tiles" and not plan["found"]


def test_refusals():
    L, R, none = ax.lib(), ctypes.byref, [None] * 5
    d = ax.ax_experts_desc_t(4, 4, 64, 32, 32, 64, 64, 32, 2, 1, 0, 0, 0, 0)
    assert L.ax_probe_experts_plan(R(d), 0, *none) == 0
    assert L.ax_probe_experts_plan(None, 0, *none) == -1
    for product in (-1, 1, 3, 8):  # no int8 codes
        assert L.ax_probe_experts_plan(R(d), product, *none) == -8
    d.N = 0
    assert L.ax_probe_experts_plan(R(d), 0, *none) == -2
    q, none = ax.ax_q4_desc_t(4, 4, 64, 32, 32, 64, 64, 2, 128, 1, 0, 0, 0), [None] * 4
    assert L.ax_probe_q4_plan(R(q), 0, *none) == 0
    assert L.ax_probe_q4_plan(None, 0, *none) == -1
    assert L.ax_probe_q4_plan(R(q), 2, *none) == -8
    q.group = 48
    assert L.ax_probe_q4_plan(R(q), 0, *none) == -8
    q.group, q.K = 128, 0
    assert L.ax_probe_q4_plan(R(q), 1, *none) == -2
