"""Waves of a workgroup of few rows and 4-bit weights (host arithmetic): sixteen only where no compute unit gets a second workgroup."""

import os

import pytest
import torch

from paper_2002_09481_amd import binding as ax

pytestmark = pytest.mark.skipif(not os.path.exists(ax.LIB_PATH), reason="libaxconv.so not built")


@pytest.mark.parametrize("rows,dtype", [(1, torch.bfloat16), (1, torch.float32), (16, torch.bfloat16), (20, torch.bfloat16), (32, torch.bfloat16)])
@pytest.mark.parametrize("K", [4096, 5120, 16384])
def test_more_workgroups_than_compute_units(rows, dtype, K):
    for N, waves in ((512, 16), (2048, 16), (4096, 16), (4112, 8), (5120, 8)):
        plan = ax.ax_probe_q4_plan(False, rows, 1, K, N, dtype=dtype)
        assert plan["kernel"] == "few" and plan["tile"][1] == 16 and plan["waves"] == waves, (N, plan)
    assert ax.ax_probe_q4_plan(False, rows, 1, 2048, 2048, dtype=dtype)["waves"] == 8
