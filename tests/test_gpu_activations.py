"""The activations by themselves: products with one, so that the value in front is exact, against 64-bit forms.

Bounds, relative, in units of u = 2^-24.  float32 results: exp(-z^2 / 2) 3.5 (the instruction two, its argument and correction the
rest), the reciprocal 1.5 times a slope of at most 1.6, the polynomial 3, its fit 0.3, four products, one minus the tail 1: 14.
silu: exponential 3, one plus it and its reciprocal 2, two products: 8.  Slopes are sums of two such terms: 16 of their sizes.
bf16 results: the short form's 1.2e-4 (silu: 1.2e-5), and the rounding of the result."""

import math

import pytest
import torch

import ff_common as F
from paper_2002_09481_amd import binding as ax

pytestmark = pytest.mark.gpu
EXACT = {"gelu": 14 * F.U, "silu": 8 * F.U}
FAST = {"gelu": 1.2e-4, "silu": 1.2e-5}


def _cdf(z):
    """(torch's ndtr is half of 1 + erf: it has no digits left in the tail.)"""
    return 0.5 * torch.special.erfc(-z * math.sqrt(0.5))


def _act(z, act):
    return z * _cdf(z) if act == "gelu" else F.act(z, act)


def _slope(z, act):
    return _cdf(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi) if act == "gelu" else F.slope(z, act)


def _values(act, n, dtype, seed):
    z = torch.rand(n, generator=F.gen(seed)) * 25 - 12.5
    z[: n // 4] = torch.rand(n // 4, generator=F.gen(seed + 1)) * 2 - 1
    if act == "silu":
        z[-n // 4:] = torch.rand(n // 4, generator=F.gen(seed + 2)) * -80
    z[:4] = torch.tensor([0.0, -1e-3, 1e-30, 5.0])
    return z.to(dtype)


def _bound(act, want, odt):
    return want.abs() * (EXACT[act] if odt == torch.float32 else F.store(odt) + FAST[act])


@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("dt,out", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f32", "bf16")])
@pytest.mark.parametrize("M,N", [(16, 1), (64, 40), (2000, 1), (2000, 264)])  # few rows; tiles
def test_values(M, N, dt, out, act):
    odt = F.DT[out]
    x, w = _values(act, M, F.DT[dt], M + N), torch.ones((1, N), dtype=F.DT[dt])
    want = _act(x.double(), act)[:, None].expand(M, N)
    y, z = ax.ax_matmul(x.cuda()[:, None], w.cuda(), act=act, out_dtype=odt, save=True)
    assert torch.equal(z.cpu(), x.to(odt)[:, None].expand(M, N))
    F.assert_within(y, want, _bound(act, want, odt), "y")
    h, _, _ = ax.ax_gated(x.cuda()[:, None], w.cuda(), (0 * w).cuda(), act=act, out_dtype=odt)
    assert not bool(h.any())
    h, _, _ = ax.ax_gated(x.cuda()[:, None], w.cuda(), w.cuda(), act=act, out_dtype=odt)
    want = (want * x.double()[:, None]).float().double()  # (1e-60 is none)
    F.assert_within(h, want, _bound(act, want, odt) + want.abs() * F.U, "h")


@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("M", [8, 2000])
def test_slopes(M, dt, act):
    dtype = F.DT[dt]
    z, one = _values(act, M, dtype, M), torch.ones((M, 1), dtype=dtype).cuda()
    zd = z.double()
    if act == "gelu":
        size = _cdf(zd) + zd.abs() * torch.exp(-zd * zd / 2) / math.sqrt(2 * math.pi)
    else:
        size = torch.special.expit(zd) * (1 + zd.abs() * torch.special.expit(-zd))
    own = size * (16 * F.U if dt == "f32" else 2 * FAST[act])
    gx, _, gb = ax.ax_matmul_backward(one, one, one[:1], z.cuda()[:, None], act=act)
    want = _slope(zd, act)[:, None]
    F.assert_within(gx, want, own[:, None] + want.abs() * F.store(dtype), "slope")
    F.assert_within(gb, want.sum(dim=0), own.sum() + size.sum() * (M / 8 + 80) * F.U, "sum of slopes")
    gx, gwg, gwu = ax.ax_gated_backward(one, one, one[:1], 0 * one[:1], z.cuda()[:, None], one, act=act)
    F.assert_within(gx, want, own[:, None] + want.abs() * F.store(dtype), "gated slope")
    gx, _, _ = ax.ax_gated_backward(one, one, 0 * one[:1], one[:1], z.cuda()[:, None], one, act=act)
    want = _act(zd, act)[:, None]
    F.assert_within(gx, want, _bound(act, want, dtype), "gated value")


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("M", [8, 300])
def test_ends(M, dt):
    """Far tails, infinities and NaN."""
    inf, nan = float("inf"), float("nan")
    z = torch.tensor([-inf, inf, nan, -1e30, 1e30, -70.0, 70.0, -20.0])
    x = torch.cat([z, torch.zeros(M - 8)])
    want = torch.tensor([0.0, inf, nan, 0.0, 1e30, 0.0, 70.0, 0.0]).to(F.DT[dt])
    if dt == "f32":
        want[4] = float(torch.tensor(1e30).bfloat16())
    low = torch.ones((1, 1), dtype=torch.bfloat16).cuda()  # (of float32 operands an infinity may give NaN)
    y = ax.ax_matmul(x.bfloat16().cuda()[:, None], low, act="gelu", out_dtype=F.DT[dt])[0].cpu().reshape(-1)[:8]
    assert torch.equal(torch.nan_to_num(y, 5.0), torch.nan_to_num(want, 5.0)) and torch.equal(torch.isnan(y), torch.isnan(want))
    y = ax.ax_matmul(x.bfloat16().cuda()[:, None], low, act="silu", out_dtype=F.DT[dt])[0].cpu().reshape(-1)
    assert bool(torch.isnan(y[2])) and y[1] == inf and y[3] == 0 and y[4] == want[4] and y[6] == 70
    one, ones = (torch.ones((n, 1), dtype=F.DT[dt]).cuda() for n in (1, M))
    s = ax.ax_matmul_backward(ones, ones, one, x.to(F.DT[dt]).cuda()[:, None], act="gelu")[0].cpu().reshape(-1)[:8]
    assert torch.equal(torch.nan_to_num(s, 5.0), torch.tensor([0.0, 1, 5, 0, 1, 0, 1, 0]).to(F.DT[dt]))
