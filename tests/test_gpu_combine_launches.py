"""Tokens' sums and their gradients with more workgroups than one launch has: what the later launches read and write.  All values are
whole numbers that bfloat16 holds, so every result is exact."""

import pytest
import torch

from paper_2002_09481_amd import binding as ax

pytestmark = pytest.mark.gpu


def _count(T, n, dtype):
    return (torch.arange(T, device="cuda", dtype=torch.int32) % n).to(dtype)


def test_sums_of_more_tokens_than_one_launch_has():
    """32 tokens a workgroup, 2^23 of those at most: the tokens are cut in halves."""
    T, n = 2 ** 28 + 5, 1009
    h = _count(n, 13, torch.bfloat16).view(n, 1)
    rows, w, r = _count(T, n, torch.int32).view(T, 1), _count(T, 7, torch.float32).view(T, 1), _count(T, 5, torch.bfloat16).view(T, 1)
    want = (_count(T, n, torch.int32) % 13).float()
    y = ax.ax_combine(h, rows)
    assert torch.equal(y.view(T), want.to(torch.bfloat16))
    del y
    want = (want * w.view(T) + r.view(T).float()).to(torch.bfloat16)
    assert torch.equal(ax.ax_combine(h, rows, w, residual=r).view(T), want)
    assert torch.equal(ax.ax_combine(h, rows, w, residual=r, y_out=r).view(T), want)


@pytest.mark.parametrize("weighted", [False, True])
def test_gradients_of_more_tokens_than_one_launch_has(weighted):
    """Four tokens a workgroup, 2^22 of those a launch."""
    T = 2 ** 24 + 5
    gy, h = _count(T, 11, torch.bfloat16).view(T, 1), _count(T, 13, torch.bfloat16).view(T, 1)
    rows = (T - 1 - torch.arange(T, device="cuda", dtype=torch.int32)).view(T, 1)
    w = _count(T, 7, torch.float32).view(T, 1) if weighted else None
    gh, gw = ax.ax_combine_backward(gy, h, rows, w)
    want = gy.float() if w is None else gy.float() * w
    assert torch.equal(gh, want.flip(0).to(torch.bfloat16)) and torch.equal(gw, gy.float() * h.float().flip(0))


def test_gradients_of_more_long_rows_than_one_launch_has():
    """A workgroup a token."""
    T, n, cols = 2 ** 22 + 5, 1009, 2049
    h = _count(n * cols, 3, torch.bfloat16).view(n, cols)
    gy = torch.empty((T, cols), dtype=torch.bfloat16, device="cuda")
    gy.copy_(_count(T, 11, torch.bfloat16).view(T, 1).expand(T, cols))
    rows = _count(T, n, torch.int32).view(T, 1)
    _, gw = ax.ax_combine_backward(gy, h, rows, gh_out=False)
    assert torch.equal(gw.view(T), _count(T, 11, torch.float32) * h.float().sum(1)[rows.view(T).long()])
