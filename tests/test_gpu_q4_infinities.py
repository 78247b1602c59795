"""Infinities and NaN in rows that meet weights of 4 bits: what the product of float32 numbers is, with both signs, and nothing of it in
other rows.  A weight of zero makes NaN of an infinity."""

import pytest
import torch

import ff_common as F
from paper_2002_09481_amd import binding as ax
from test_gpu_q4 import _sums, _way, _weights

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


def _rows(g, M, K, dtype):
    """Row, and what is put into it: a column's value."""
    x = F.randn(g, (M, K), 1.0, dtype)
    for row, put in enumerate(([], [(3, INF)], [(K - 1, -INF)], [(3, INF), (70, INF)], [(3, INF), (99, -INF)], [(40, NAN)], [(40, NAN), (41, INF)])):
        for k, v in put:
            x[row, k] = v
    return x


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,K,N", [(7, 200, 33), (16, 264, 600), (31, 200, 80), (64, 264, 130), (300, 264, 3700), (700, 200, 1650)])
def test_infinities(M, K, N, group, dt):
    g, dtype = F.gen(M + group), F.DT[dt]
    x = _rows(g, M, K, dtype)
    q, w, most = _weights(g, (N, K), group)
    way = _way(M, N, dtype=dtype)
    want, y = x.double() @ w.t(), ax.ax_matmul_q4(x.cuda(), q).double().cpu()
    sound = torch.isfinite(want)
    assert torch.equal(sound[:, 0], torch.tensor([row not in (1, 2, 3, 4, 5, 6) for row in range(M)])) and torch.equal(torch.isfinite(y), sound)
    if way == "tiles" and dtype == torch.bfloat16:  # (24 is taken off again, an infinity from another)
        assert bool((torch.isnan(y) | (y == want))[~sound].all())
    else:
        assert torch.equal(torch.isnan(y), torch.isnan(want)) and bool((y == want)[torch.isinf(want)].all())
    x[~sound[:, 0]] = 0  # (whole rows)
    xd = x.double()
    bound = _sums(xd, w, most, K, way, dtype) + (xd @ w.t()).abs() * F.store(dtype)
    F.assert_within(torch.where(sound, y, 0.0), xd @ w.t(), bound)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("M", [7, 40])
def test_infinities_of_a_gated_pair(M, dt):
    g, dtype = F.gen(M), F.DT[dt]
    x = _rows(g, M, 200, dtype)
    (q, w, _), (qu, wu, _) = _weights(g, (48, 200), 64), _weights(g, (48, 200), 64)
    xd = x.double()
    want = torch.relu(xd @ w.t()) * (xd @ wu.t())
    h = ax.ax_gated_q4(x.cuda(), q, qu, act="relu").double().cpu()
    assert torch.equal(torch.isnan(h), torch.isnan(want)) and torch.equal(torch.isinf(h), torch.isinf(want))
    assert bool((h == want)[torch.isinf(want)].all())
