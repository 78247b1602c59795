"""float32 products: the three bf16 pieces of an operand, one product at a time (a contraction over one element).

Bound: what the pieces leave out is at most 2^-24 (1 + 2^-8) of the product; the six products that are kept are exact and added
smallest first, so that the last addition alone rounds on the result's scale, by one unit of 2^-23 at most, the others 2^-8 of it."""

import pytest
import torch

import ff_common as F
from paper_2002_09481_amd import binding as ax

pytestmark = pytest.mark.gpu
BOUND = (1 + 2.0 ** -8) * F.U + 2 * F.U * (1 + 2.0 ** -6)


def _long(g, n, spread):
    """Floats from 1 on whose significands use all their bits, `spread` bits of them at random, both ends of that among them."""
    bits = 0x3F800000 + torch.randint(0, 1 << spread, (n,), generator=g, dtype=torch.int32)
    bits[0], bits[1] = 0x3F80FFFF, 0x3F80FFFF + (1 << (spread - 1) if spread > 17 else 0)
    return bits.view(torch.float32)


@pytest.mark.parametrize("spread", [17, 23])
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("M,N", [(32, 520), (300, 520)])  # few rows, tiles
def test_products_of_one_sign(M, N, transposed, spread):
    g = F.gen(M + spread)
    x, w = _long(g, M, spread), _long(g, N, spread)
    want = x.double()[:, None] * w.double()
    y, _ = ax.ax_matmul(x.cuda()[:, None], w.cuda()[:, None] if transposed else w.cuda()[None], transposed=transposed)
    F.assert_within(y, want, want.abs() * BOUND, "y")
    gx, gw, _ = ax.ax_matmul_backward(x.cuda()[:1, None].expand(1, 1).contiguous(), w.cuda()[None], w.cuda()[:, None])
    want = x[0].double() * w.double()
    F.assert_within(gx, want[None], want[None].abs() * BOUND, "gx")
    F.assert_within(gw, want[:, None], want[:, None].abs() * BOUND, "gw")


@pytest.mark.parametrize("M", [4, 200])
def test_values_next_to_the_largest(M):
    """They would round to infinity in 16 bits."""
    bits = torch.tensor([0x7F7FFFFF, 0x7F7F8000, 0x7F7F7FFF, 0x7F7FC001, 0x7F000000, 0x7F7F0001], dtype=torch.int64)
    x = torch.cat([bits, bits + 0x80000000 - (1 << 32)]).to(torch.int32).view(torch.float32)
    w = torch.tensor([0.5, -0.5, 0.25, 2.0 ** -100, 1.0], dtype=torch.float32)
    xs = x.repeat(-(-M // x.numel()))[:M]
    want = xs.double()[:, None] * w.double()
    y, _ = ax.ax_matmul(xs.cuda()[:, None], w.cuda()[None])
    F.assert_within(y, want, want.abs() * BOUND)
    y, _ = ax.ax_matmul(w.cuda()[:, None], xs.cuda()[None])
    F.assert_within(y, want.t(), want.t().abs() * BOUND)
