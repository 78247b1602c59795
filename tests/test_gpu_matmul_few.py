"""Products of few rows: contractions cut into slices, rows that start inside a word, 17 to 32 rows of every type."""

import pytest
import torch

import ff_common as F
from paper_2002_09481_amd import binding as ax

pytestmark = pytest.mark.gpu

# (M, K, N): few columns of a long contraction, contractions that end inside a slice, a step or a lane's share, odd rows
SIZES = [(1, 8192, 16), (8, 6117, 130), (16, 4097, 33), (17, 8192, 7), (31, 5003, 40), (32, 4096, 257), (32, 130, 1001), (29, 2051, 600)]


def _placed(t, offset):
    """t on the device, its first element `offset` elements into a buffer."""
    buf = torch.zeros(t.numel() + offset, dtype=t.dtype, device="cuda")
    buf[offset:] = t.reshape(-1).cuda()
    return buf[offset:].view(t.shape)


def _bound(zd, zb, name, dtype):
    yd = F.act(zd, name)
    return yd, zb * F.ACT_LIP + yd.abs() * F.ACT_REL + F.U * zd.abs()


@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", SIZES)
def test_forward(M, K, N, dt, transposed, offset):
    dtype, g = F.DT[dt], F.gen(M * 7 + K * 3 + N)
    x, w = F.randn(g, (M, K), 1.0, dtype), F.randn(g, (N, K) if transposed else (K, N), K ** -0.5, dtype)
    b, r = F.randn(g, (N,), 1.0, dtype), F.randn(g, (M, N), 1.0, dtype)
    wd = w.double().t() if transposed else w.double()
    zd, zb = x.double() @ wd + b.double(), x.double().abs() @ wd.abs() * F.sum_bound(K, dt == "f32")
    zb = zb + F.U * (zd.abs() + b.double().abs())
    xc, wc = _placed(x, offset), _placed(w, offset)
    y, z = ax.ax_matmul(xc, wc, bias=b.cuda(), residual=r.cuda(), act="silu", transposed=transposed, save=True)
    F.assert_within(z, zd, zb + zd.abs() * F.store(dtype), "z")
    yd, bound = _bound(zd, zb, "silu", dtype)
    yd = yd + r.double()
    F.assert_within(y, yd, bound + 2 * F.U * (yd.abs() + r.double().abs()) + yd.abs() * F.store(dtype), "y")
    again = ax.ax_matmul(x.cuda(), w.cuda(), bias=b.cuda(), residual=r.cuda(), act="silu", transposed=transposed, save=True)
    assert torch.equal(again[0], y) and torch.equal(again[1], z)  # the placement changes no bit


@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", SIZES)
def test_gated(M, K, N, dt, offset):
    dtype, g = F.DT[dt], F.gen(M + K * 3 + N)
    x, ws = F.randn(g, (M, K), 1.0, dtype), [F.randn(g, (K, N), K ** -0.5, dtype) for _ in range(2)]
    gd, ud = (x.double() @ w.double() for w in ws)
    gb, ub = (x.double().abs() @ w.double().abs() * F.sum_bound(K, dt == "f32") for w in ws)
    h, gc, uc = ax.ax_gated(_placed(x, offset), *(_placed(w, offset) for w in ws), act="gelu", save=True)
    F.assert_within(gc, gd, gb + gd.abs() * F.store(dtype), "g")
    F.assert_within(uc, ud, ub + ud.abs() * F.store(dtype), "u")
    ad, ab = _bound(gd, gb, "gelu", dtype)
    hd = ad * ud
    F.assert_within(h, hd, ab * (ud.abs() + ub) + ad.abs() * ub + hd.abs() * (2 * F.U + F.store(dtype)), "h")


@pytest.mark.parametrize("offset", [0, 1, 2, 3])
@pytest.mark.parametrize("M,K,N", SIZES)
def test_codes(M, K, N, offset):
    g = F.gen(M + K + N)
    mats = [torch.randint(-127, 128, (rows, K), generator=g, dtype=torch.int8) for rows in (M, N, N)]
    x, w, w2 = mats
    xs, ws, ws2 = (torch.rand(t.shape[0], generator=g) * 0.02 + 1e-3 for t in mats)
    a, a2 = ((x.double() @ v.double().t()) * xs.double()[:, None] * s.double() for v, s in ((w, ws), (w2, ws2)))
    dev = [_placed(x, offset), xs.cuda(), _placed(w, offset), ws.cuda()]
    y = ax.ax_matmul_q8(*dev, out_dtype=torch.float32)
    F.assert_within(y, a, a.abs() * (4 * F.U + F.store(torch.float32)), "sum")
    h = ax.ax_gated_q8(*dev, _placed(w2, offset), ws2.cuda(), act="silu", out_dtype=torch.float32)
    hd = F.act(a, "silu") * a2
    F.assert_within(h, hd, 8 * F.U * (F.ACT_LIP * a.abs() * a2.abs() + hd.abs()) + hd.abs() * (F.ACT_REL + F.store(torch.float32)), "gated")


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", [(8, 616, 5003), (16, 40, 8192), (1, 33, 4099), (32, 100, 4097)])
def test_gated_input_gradient(M, K, N, dt):
    """The input's gradient contracts over the long side of both projections, one after the other."""
    dtype, g = F.DT[dt], F.gen(M + K + N)
    x, ws = F.randn(g, (M, K), 1.0, dtype), [F.randn(g, (K, N), K ** -0.5, dtype) for _ in range(2)]
    gh, gp, up = (F.randn(g, (M, N), 1.0, dtype) for _ in range(3))
    gx, _, _ = ax.ax_gated_backward(gh.cuda(), x.cuda(), *(w.cuda() for w in ws), gp.cuda(), up.cuda(), act="silu")
    hd = gh.double()
    parts = [hd * up.double() * F.slope(gp.double(), "silu"), hd * F.act(gp.double(), "silu")]
    sizes = [hd.abs() * up.double().abs(), hd.abs() * gp.double().abs()]  # |slope| and |act / z| are at most 1.13
    want, bound = 0, 0
    for p, s, w in zip(parts, sizes, ws):
        one = 32 * F.U * 1.13 * s + (p.abs() * 2.0 ** -8 * 1.01 if dt == "bf16" else 0)
        want = want + p @ w.double().t()
        bound = bound + one @ w.double().abs().t() + p.abs() @ w.double().abs().t() * F.sum_bound(2 * N, dt == "f32")
    F.assert_within(gx, want, bound + want.abs() * F.store(dtype), "gx")


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", [(12, 2048, 40), (13, 70, 300), (16, 2048, 2048), (17, 1030, 1021), (32, 1024, 1024), (31, 513, 2100), (33, 1024, 1030)])
def test_gradients(M, K, N, dt, transposed):
    dtype, g = F.DT[dt], F.gen(M + 5 * K + N)
    x, w = F.randn(g, (M, K), 1.0, dtype), F.randn(g, (N, K) if transposed else (K, N), K ** -0.5, dtype)
    gy, z = F.randn(g, (M, N), 1.0, dtype), F.randn(g, (M, N), 1.5, dtype)
    wd = w.double().t() if transposed else w.double()
    gz = gy.double() * F.slope(z.double(), "silu")
    gx, gw, gb = ax.ax_matmul_backward(gy.cuda(), x.cuda(), w.cuda(), z.cuda(), act="silu", transposed=transposed)
    one = 24 * F.U * gy.double().abs() + (gz.abs() * 2.0 ** -8 if dt == "bf16" else 0)
    want = gz @ wd.t()
    F.assert_within(gx, want, one @ wd.t().abs() + gz.abs() @ wd.t().abs() * F.sum_bound(N, dt == "f32") + want.abs() * F.store(dtype), "gx")
    xt = x.double().t()
    want, bound = xt @ gz, xt.abs() @ one + xt.abs() @ gz.abs() * F.sum_bound(M, dt == "f32")
    bound = bound + want.abs() * F.store(dtype)
    F.assert_within(gw, want.t() if transposed else want, bound.t() if transposed else bound, "gw")
    F.assert_within(gb, gz.sum(dim=0), (24 * F.U * gy.double().abs()).sum(dim=0) + gz.abs().sum(dim=0) * (M / 8 + 80) * F.U, "gb")


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("M,K,N", [(33, 512, 130), (48, 6000, 64), (63, 333, 1001), (64, 2052, 96), (64, 2051, 96), (65, 512, 64)])
def test_bands_of_rows(M, K, N, transposed):
    """float32 rows of several workgroups, with and without slices; one row more goes through tiles."""
    g = F.gen(M + K + N)
    x, w, w2 = F.randn(g, (M, K)), F.randn(g, (N, K) if transposed else (K, N), K ** -0.5), F.randn(g, (K, N), K ** -0.5)
    r, wd = F.randn(g, (M, N)), w.double().t() if transposed else w.double()
    zd, zb = x.double() @ wd, x.double().abs() @ wd.abs() * F.sum_bound(K, True)
    y, z = ax.ax_matmul(x.cuda(), w.cuda(), residual=r.cuda(), act="silu", transposed=transposed, save=True)
    F.assert_within(z, zd, zb + zd.abs() * F.store(torch.float32), "z")
    yd, bound = _bound(zd, zb, "silu", torch.float32)
    yd = yd + r.double()
    F.assert_within(y, yd, bound + 2 * F.U * (yd.abs() + r.double().abs()) + yd.abs() * F.store(torch.float32), "y")
    if not transposed:
        ud, ub = x.double() @ w2.double(), x.double().abs() @ w2.double().abs() * F.sum_bound(K, True)
        h, _, u = ax.ax_gated(x.cuda(), w.cuda(), w2.cuda(), act="silu", save=True)
        F.assert_within(u, ud, ub + ud.abs() * F.store(torch.float32), "u")
        ad, ab = _bound(zd, zb, "silu", torch.float32)
        F.assert_within(h, ad * ud, ab * (ud.abs() + ub) + ad.abs() * ub + (ad * ud).abs() * (2 * F.U + F.store(torch.float32)), "h")
