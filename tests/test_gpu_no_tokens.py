"""Steps of blocks without a token (a batch that is empty on one rank): gradients of zero, and the parameters' gradients skipped."""

import pytest
import torch

import ff_common as F
from paper_2002_09481_amd import binding as ax
from paper_2002_09481_amd.feedforward import ExpertsFeedForward, FeedForward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("experts", [False, True])
def test_a_step_without_tokens(experts, dt):
    b = ExpertsFeedForward(64, 96, 5, 2, dtype=F.DT[dt]) if experts else FeedForward(64, 96, dtype=F.DT[dt])
    for t in b.grads.values():
        t.fill_(7)
    x = torch.empty((0, 64), device="cuda", dtype=F.DT[dt])
    assert b.forward(x, train=True).shape == (0, 64) and b.backward(x).shape == (0, 64)
    assert not any(bool(t.any()) for t in b.grads.values())
    before = {n: t.clone() for n, t in b.master.items()}
    b.step(1e-2)
    assert all(torch.equal(t, before[n]) for n, t in b.master.items())


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_gradients_of_no_rows_by_experts(dt):
    dtype = F.DT[dt]
    x, y, w = torch.empty((0, 64), device="cuda", dtype=dtype), torch.empty((0, 96), device="cuda", dtype=dtype), torch.ones((5, 64, 96), device="cuda", dtype=dtype)
    o, rows, p = torch.zeros(6, dtype=torch.int32, device="cuda"), torch.empty((0, 2), dtype=torch.int32, device="cuda"), torch.empty((0, 2), device="cuda")
    for skip in (False, None):
        gx, gw = ax.ax_matmul_experts_backward(y, x, w, o, gw_out=skip)
        assert gx.shape == (0, 64) and (gw is None if skip is False else not bool(gw.any()))
        gx, *gws = ax.ax_gated_experts_backward(y, x, w, w, y, y, o, gwg_out=skip, gwu_out=skip)
        assert gx.shape == (0, 64) and all(g is None if skip is False else not bool(g.any()) for g in gws)
    for h in (y, torch.empty((3, 96), device="cuda", dtype=dtype)):
        gh, gweights = ax.ax_combine_backward(y, h, rows, p)
        assert gh.shape == h.shape and gweights.shape == (0, 2)
        assert ax.ax_combine_backward(y, h, rows, p, gh_out=False)[1].shape == (0, 2)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_gradients_of_no_rows(dt):
    dtype = F.DT[dt]
    x, y, w = torch.empty((0, 64), device="cuda", dtype=dtype), torch.empty((0, 96), device="cuda", dtype=dtype), torch.ones((64, 96), device="cuda", dtype=dtype)
    for skip in (False, None):
        gx, *rest = ax.ax_matmul_backward(y, x, w, gw_out=skip, gb_out=skip)
        assert gx.shape == (0, 64) and all(g is None if skip is False else not bool(g.any()) for g in rest)
        gx, *rest = ax.ax_gated_backward(y, x, w, w, y, y, gwg_out=skip, gwu_out=skip)
        assert gx.shape == (0, 64) and all(g is None if skip is False else not bool(g.any()) for g in rest)
        gx, gw = ax.ax_rmsnorm_backward(x, x, w[:, 0].contiguous(), torch.empty(0, device="cuda"), gw_out=skip)
        assert gx.shape == (0, 64) and (gw is None if skip is False else not bool(gw.any()))
