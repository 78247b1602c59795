"""Gradients of no rows: the arrays that have a row for each are NULL then, which is no reason to refuse the call (no GPU needed)."""

import ctypes
import os

import pytest

from paper_2002_09481_amd import binding as ax
from test_experts_refusals import P, combine, experts
from test_feedforward_refusals import mm, norm

pytestmark = pytest.mark.skipif(not os.path.exists(ax.LIB_PATH), reason="libaxconv.so not built")
R = ctypes.byref


def test_tokens_sums():
    L = ax.lib()
    for h_rows in (0, 5):
        d = combine(tokens=0, h_rows=h_rows)
        assert L.ax_combine_backward(R(d), *[None] * 7) == 0
        assert L.ax_combine_backward(R(d), *[None] * 4, P, None, None) == 0
    assert L.ax_combine_backward(R(combine(tokens=-1)), *[None] * 7) == -2


def test_products_by_experts():
    L, d = ax.lib(), experts(rows=0, x_rows=0)
    assert L.ax_matmul_experts_backward(R(d), *[None] * 9, 0, None) == 0
    assert L.ax_gated_experts_backward(R(d), *[None] * 12, 0, None) == 0
    assert L.ax_gated_experts_backward(R(d), *[None] * 9, P, None, None, 0, None) == -1  # one weight's gradient without the other's


def test_norm_and_whole_products():
    L, d = ax.lib(), mm(M=0)
    assert L.ax_rmsnorm_backward(R(norm(rows=0)), *[None] * 8, 0, None) == 0
    assert L.ax_matmul_backward(R(d), *[None] * 8, 0, None) == 0
    assert L.ax_gated_backward(R(d), *[None] * 10, 0, None) == 0
    assert L.ax_gated_backward(R(d), *[None] * 7, P, None, None, 0, None) == -1
