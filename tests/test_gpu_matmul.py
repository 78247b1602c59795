"""Matrix products with their epilogue, the gated block, and their gradients against 64-bit forms, at sizes either side of the
tiles, odd ones, every operand layout and placement."""

import pytest
import torch

import ff_common as F
from paper_2002_09481_amd import binding as ax

pytestmark = pytest.mark.gpu

ACTS = ["none", "relu", "silu", "gelu"]
# (M, K, N): single elements, one token, odd everywhere, tile edges, long sums in slices, several tiles a side
SIZES = [(1, 1, 1), (1, 256, 512), (3, 7, 5), (1, 4096, 136), (17, 520, 264), (33, 64, 129), (130, 193, 257), (64, 8192, 96),
         (128, 128, 128), (257, 320, 513), (300, 72, 1000), (1000, 333, 136), (2, 2049, 2050), (16, 1000, 3)]


def _product(x, w):
    return x @ w, x.abs() @ w.abs()


def _check(y, z, zd, zb, name, r, dtype, what=""):
    if z is not None:
        F.assert_within(z, zd, zb + zd.abs() * F.store(dtype), what + " z")
    yd = F.act(zd, name)
    bound = zb * F.ACT_LIP + yd.abs() * F.ACT_REL + F.U * zd.abs()
    if r is not None:
        yd = yd + r
        bound = bound + 2 * F.U * (yd.abs() + r.abs())
    F.assert_within(y, yd, bound + yd.abs() * F.store(dtype), what + " y")


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", SIZES)
def test_forward(M, K, N, dt, transposed):
    dtype, g = F.DT[dt], F.gen(M * 7 + K * 3 + N)
    x, w = F.randn(g, (M, K), 1.0, dtype), F.randn(g, (N, K) if transposed else (K, N), K ** -0.5, dtype)
    b, r = F.randn(g, (N,), 1.0, dtype), F.randn(g, (M, N), 1.0, dtype)
    wd = w.double().t() if transposed else w.double()
    zd, size = _product(x.double(), wd)
    xc, wc, bc, rc = x.cuda(), w.cuda(), b.cuda(), r.cuda()
    y, z = ax.ax_matmul(xc, wc, transposed=transposed)
    assert z is None
    zb = size * F.sum_bound(K, dt == "f32")
    _check(y, None, zd, zb, "none", None, dtype)
    zd, zb = zd + b.double(), zb + F.U * (zd.abs() + b.double().abs())
    for i, name in enumerate(ACTS):
        y, z = ax.ax_matmul(xc, wc, bias=bc, residual=rc if i % 2 else None, act=name, transposed=transposed, save=True)
        _check(y, z, zd, zb, name, r.double() if i % 2 else None, dtype, name)
    if dt == "bf16":  # float32 results of bf16 operands: nothing but the sum's own rounding
        y, _ = ax.ax_matmul(xc, wc, bias=bc.float(), transposed=transposed, out_dtype=torch.float32)
        _check(y, None, zd, zb, "none", None, torch.float32, "f32 out")


def _codes(g, rows, cols):
    c = torch.randint(-127, 128, (rows, cols), generator=g, dtype=torch.int8)
    return c, torch.rand(rows, generator=g) * 0.02 + 1e-3


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", SIZES + [(5, 20000, 40)])
def test_codes(M, K, N, out):
    dtype, g = F.DT[out], F.gen(M + K + N)
    (x, xs), (w, ws), (w2, ws2) = _codes(g, M, K), _codes(g, N, K), _codes(g, N, K)
    b, r = F.randn(g, (N,), 1.0, dtype), F.randn(g, (M, N), 1.0, dtype)
    a, a2 = ((x.double() @ v.double().t()) * xs.double()[:, None] * s.double() for v, s in ((w, ws), (w2, ws2)))
    dev = [t.cuda() for t in (x, xs, w, ws)]
    y = ax.ax_matmul_q8(*dev, out_dtype=dtype)
    F.assert_within(y, a, a.abs() * (4 * F.U + F.store(dtype)), "sum")  # the sum is exact: two products, one conversion
    for name in ACTS:
        y = ax.ax_matmul_q8(*dev, bias=b.cuda(), residual=r.cuda(), act=name, out_dtype=dtype)
        _check(y, None, a + b.double(), 6 * F.U * (a.abs() + b.double().abs()), name, r.double(), dtype, name)
        h = ax.ax_gated_q8(*dev, w2.cuda(), ws2.cuda(), act=name, out_dtype=dtype)
        hd = F.act(a, name) * a2
        F.assert_within(h, hd, 8 * F.U * (F.ACT_LIP * a.abs() * a2.abs() + hd.abs()) + hd.abs() * (F.ACT_REL + F.store(dtype)), "gated " + name)


def test_codes_at_their_limits():
    x = torch.full((3, 131071), -128, dtype=torch.int8, device="cuda")
    one = torch.ones(3, device="cuda")
    y = ax.ax_matmul_q8(x, one, x, one, out_dtype=torch.float32)
    assert torch.equal(y, torch.full((3, 3), float(131071 * 16384), device="cuda"))


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", [(1, 1, 1), (3, 7, 5), (1, 264, 520), (130, 193, 257), (700, 72, 64), (257, 320, 128), (64, 40, 1030)])
def test_gradients(M, K, N, dt, transposed, act):
    dtype, g = F.DT[dt], F.gen(M + 5 * K + N)
    x, w = F.randn(g, (M, K), 1.0, dtype), F.randn(g, (N, K) if transposed else (K, N), K ** -0.5, dtype)
    gy, z = F.randn(g, (M, N), 1.0, dtype), F.randn(g, (M, N), 1.5, dtype)
    wd = w.double().t() if transposed else w.double()
    gz = gy.double() * F.slope(z.double(), act)
    out = ax.ax_matmul_backward(gy.cuda(), x.cuda(), w.cuda(), z.cuda() if act != "none" else None, act=act, transposed=transposed)
    # gz itself: a slope and a product; bf16: rounded for the products
    one = 24 * F.U * gy.double().abs() + (gz.abs() * 2.0 ** -8 if dt == "bf16" and act != "none" else 0)
    f32 = dt == "f32"
    want = gz @ wd.t()
    F.assert_within(out[0], want, one @ wd.t().abs() + gz.abs() @ wd.t().abs() * F.sum_bound(N, f32) + want.abs() * F.store(dtype), "gx")
    want = x.double().t() @ gz
    bound = x.double().t().abs() @ one + x.double().t().abs() @ gz.abs() * F.sum_bound(M, f32) + want.abs() * F.store(dtype)
    F.assert_within(out[1], want.t().contiguous() if transposed else want, bound.t() if transposed else bound, "gw")
    F.assert_within(out[2], gz.sum(dim=0), (24 * F.U * gy.double().abs()).sum(dim=0) + gz.abs().sum(dim=0) * (M / 8 + 80) * F.U, "gb")
    again = [ax.ax_matmul_backward(gy.cuda(), x.cuda(), w.cuda(), z.cuda() if act != "none" else None, act=act, transposed=transposed,
                                   **{k: False for j, k in enumerate(("gx_out", "gw_out", "gb_out")) if j != i})[i] for i in range(3)]
    assert all(torch.equal(a, b) for a, b in zip(again, out))


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,F_", [(1, 1, 1), (3, 7, 5), (1, 520, 264), (17, 64, 300), (257, 320, 136), (130, 193, 259)])
def test_gated(M, K, F_, dt, act):
    dtype, g = F.DT[dt], F.gen(M + K + 9 * F_)
    x, wg, wu = F.randn(g, (M, K), 1.0, dtype), F.randn(g, (K, F_), K ** -0.5, dtype), F.randn(g, (K, F_), K ** -0.5, dtype)
    f32 = dt == "f32"
    h, gp, up = ax.ax_gated(x.cuda(), wg.cuda(), wu.cuda(), act=act, save=True)
    gd, gs = _product(x.double(), wg.double())
    ud, us = _product(x.double(), wu.double())
    s = F.sum_bound(K, f32)
    F.assert_within(gp, gd, gs * s + gd.abs() * F.store(dtype), "g")
    F.assert_within(up, ud, us * s + ud.abs() * F.store(dtype), "u")
    hd = F.act(gd, act) * ud
    hb = F.ACT_LIP * gs * s * (ud.abs() + us * s) + F.act(gd, act).abs() * us * s + hd.abs() * (F.ACT_REL + 2 * F.U + F.store(dtype))
    F.assert_within(h, hd, hb, "h")
    assert torch.equal(h, ax.ax_gated(x.cuda(), wg.cuda(), wu.cuda(), act=act)[0])

    gh, gv, uv = (F.randn(g, (M, F_), 1.0, dtype) for _ in range(3))
    out = ax.ax_gated_backward(gh.cuda(), x.cuda(), wg.cuda(), wu.cuda(), gv.cuda(), uv.cuda(), act=act)
    gg, gu = gh.double() * uv.double() * F.slope(gv.double(), act), gh.double() * F.act(gv.double(), act)
    low = 0 if f32 else 2.0 ** -8
    bg = 24 * F.U * (gh.double() * uv.double()).abs() + gg.abs() * low
    bu = 24 * F.U * (gh.double() * gv.double()).abs() + gu.abs() * low
    wgt, wut, xt = wg.double().t(), wu.double().t(), x.double().t()
    want = gg @ wgt + gu @ wut
    F.assert_within(out[0], want, bg @ wgt.abs() + bu @ wut.abs() + (gg.abs() @ wgt.abs() + gu.abs() @ wut.abs()) * F.sum_bound(2 * F_, f32) +
                    want.abs() * F.store(dtype), "gx")
    for o, v, bv, n in ((out[1], gg, bg, "gwg"), (out[2], gu, bu, "gwu")):
        want = xt @ v
        F.assert_within(o, want, xt.abs() @ bv + xt.abs() @ v.abs() * F.sum_bound(M, f32) + want.abs() * F.store(dtype), n)
    only = ax.ax_gated_backward(gh.cuda(), x.cuda(), wg.cuda(), wu.cuda(), gv.cuda(), uv.cuda(), act=act, gx_out=False)
    assert only[0] is None and torch.equal(only[1], out[1]) and torch.equal(only[2], out[2])
    only = ax.ax_gated_backward(gh.cuda(), x.cuda(), wg.cuda(), wu.cuda(), gv.cuda(), uv.cuda(), act=act, gwg_out=False, gwu_out=False)
    assert only[1] is None and torch.equal(only[0], out[0])


def test_gradients_against_differences():
    """A loss of matmul and of the gated block along one direction of all their inputs: central differences of the 64-bit form."""
    g = F.gen(21)
    M, K, N = 6, 20, 12
    x, wg, wu, wd, b, c = (torch.randn(s, generator=g) for s in ((M, K), (K, N), (K, N), (N, K), (K,), (M, K)))
    d = [torch.randn(t.shape, generator=g).double() for t in (x, wg, wu, wd, b)]

    def loss(e):
        X, G, U_, D, B = (t.double() + e * v for t, v in zip((x, wg, wu, wd, b), d))
        h = F.act(X @ G, "silu") * (X @ U_)
        return float((c.double() * F.act(h @ D + B, "gelu")).sum())

    X, G, U_, D, B, C = (t.cuda() for t in (x, wg, wu, wd, b, c))
    h, gp, up = ax.ax_gated(X, G, U_, save=True)
    _, z = ax.ax_matmul(h, D, bias=B, act="gelu", save=True)
    gh, gd, gb = ax.ax_matmul_backward(C, h, D, z, act="gelu")
    gx, gg, gu = ax.ax_gated_backward(gh, X, G, U_, gp, up)
    terms = [(o.cpu().double() * v) for o, v in zip((gx, gg, gu, gd, gb), d)]
    got, size = sum(float(t.sum()) for t in terms), sum(float(t.abs().sum()) for t in terms)
    e = 1e-5
    slope = (loss(e) - loss(-e)) / (2 * e)
    third = abs(loss(1e-2) - 2 * loss(5e-3) + 2 * loss(-5e-3) - loss(-1e-2)) / (2 * 5e-3 ** 3)
    # differences: their third-order term and the 64-bit losses' rounding; gradients: three float32 stages
    assert abs(got - slope) <= e * e * third + 1e-15 * size / e + size * 200 * F.U


@pytest.mark.parametrize("dt", ["f32", "bf16", "q8"])
@pytest.mark.parametrize("offset,pad", [(0, 16), (1, 6), (8, 0), (5, 11)])
def test_pitches_and_places(dt, offset, pad):
    """Operands and outputs inside wider buffers, at any element: the bits of the contiguous call, nothing else written."""
    g, M, K, N = F.gen(4), 70, 144, 208
    inner = lambda t: t[:, offset:offset + t.shape[1] - offset - pad]  # noqa: E731
    wide = lambda r, c, dtype: F.randn(g, (r, c + offset + pad), 1.0, dtype).cuda()  # noqa: E731
    odt = torch.bfloat16 if dt == "q8" else F.DT[dt]
    r, ybuf = inner(wide(M, N, odt)), wide(M, N, odt)
    y = inner(ybuf)
    old = ybuf.clone()
    if dt == "q8":
        x, w = (torch.randint(-127, 128, (n, K + offset + pad), generator=g, dtype=torch.int8).cuda() for n in (M, N))
        x, w = inner(x), inner(w)
        xs, ws = torch.rand(M, generator=g).cuda(), torch.rand(N, generator=g).cuda()
        ref = ax.ax_matmul_q8(x.contiguous(), xs, w.contiguous(), ws, residual=r.contiguous())
        ax.ax_matmul_q8(x, xs, w, ws, residual=r, y_out=y)
        assert torch.equal(ax.ax_gated_q8(x, xs, w, ws, w, ws),
                           ax.ax_gated_q8(x.contiguous(), xs, w.contiguous(), ws, w.contiguous(), ws))
    else:
        x, w, w2 = inner(wide(M, K, odt)), inner(wide(K, N, odt)), inner(wide(K, N, odt))
        ref, z = ax.ax_matmul(x.contiguous(), w.contiguous(), residual=r.contiguous(), act="silu", save=True)
        ax.ax_matmul(x, w, residual=r, act="silu", y_out=y)
        out = ax.ax_matmul_backward(r, x, w, z, act="silu")
        want = ax.ax_matmul_backward(r.contiguous(), x.contiguous(), w.contiguous(), z, act="silu")
        assert all(torch.equal(a, b) for a, b in zip(out, want)) and out[0].stride() == x.stride()
        out = ax.ax_matmul_backward(r, x, w)  # (gy is an operand itself)
        want = ax.ax_matmul_backward(r.contiguous(), x.contiguous(), w.contiguous())
        assert all(torch.equal(a, b) for a, b in zip(out, want))
        assert torch.equal(ax.ax_gated(x, w, w2)[0], ax.ax_gated(x.contiguous(), w.contiguous(), w2.contiguous())[0])
        out = ax.ax_gated_backward(r, x, w, w2, z, z)
        want = ax.ax_gated_backward(r.contiguous(), x.contiguous(), w.contiguous(), w2.contiguous(), z, z)
        assert all(torch.equal(a, b) for a, b in zip(out, want))
    assert torch.equal(y, ref)
    inner(ybuf)[:] = inner(old)
    assert torch.equal(ybuf, old)


@pytest.mark.parametrize("M,K,N", [(3, 64, 40), (40, 4096, 72), (300, 72, 264)])
def test_result_in_the_place_of_the_residual(M, K, N):
    g = F.gen(M)
    x, w, r = F.randn(g, (M, K), 1.0, torch.bfloat16).cuda(), F.randn(g, (K, N), K ** -0.5, torch.bfloat16).cuda(), F.randn(g, (M, N), 1.0, torch.bfloat16).cuda()
    want, _ = ax.ax_matmul(x, w, residual=r, act="gelu")
    y, _ = ax.ax_matmul(x, w, residual=r, act="gelu", y_out=r)
    assert y is r and torch.equal(r, want)


# both sides of the bounds between the kernel of few rows and the tiles, of its own fragments of 16 rows and 16, 32 or 64
# columns, and of its waves' turns along the contraction
@pytest.mark.parametrize("dt", ["f32", "bf16", "q8"])
@pytest.mark.parametrize("M", [2, 15, 16, 17, 31, 32, 33])
@pytest.mark.parametrize("K,N", [(1, 17), (30, 33), (129, 16), (2048, 48), (2050, 31), (4100, 70), (72, 8200), (40, 16400)])
def test_few_rows(M, K, N, dt):
    g = F.gen(M * K + N)
    if dt == "q8":
        (x, xs), (w, ws) = _codes(g, M, K), _codes(g, N, K)
        y = ax.ax_matmul_q8(x.cuda(), xs.cuda(), w.cuda(), ws.cuda(), out_dtype=torch.float32)
        a = (x.double() @ w.double().t()) * xs.double()[:, None] * ws.double()
        F.assert_within(y, a, a.abs() * 5 * F.U)
        h = ax.ax_gated_q8(x.cuda(), xs.cuda(), w.cuda(), ws.cuda(), w.cuda(), ws.cuda(), act="relu", out_dtype=torch.float32)
        F.assert_within(h, torch.relu(a) * a, a * a * 12 * F.U)
        return
    dtype = F.DT[dt]
    x, w, wt = F.randn(g, (M, K), 1.0, dtype), F.randn(g, (K, N), K ** -0.5, dtype), F.randn(g, (N, K), K ** -0.5, dtype)
    b = F.randn(g, (N,), 1.0, torch.float32)
    for v, vd, t in ((w, w.double(), False), (wt, wt.double().t(), True)):
        zd, size = _product(x.double(), vd)
        zd = zd + b.double()
        y, z = ax.ax_matmul(x.cuda(), v.cuda(), bias=b.cuda(), transposed=t, act="silu", out_dtype=torch.float32, save=True)
        zb = size * F.sum_bound(K, dt == "f32") + 2 * F.U * (zd.abs() + b.double().abs())
        F.assert_within(z, zd, zb, "z")
        F.assert_within(y, F.act(zd, "silu"), zb * F.ACT_LIP + F.act(zd, "silu").abs() * F.ACT_REL, "y")
        gy = F.randn(g, (M, N), 1.0, dtype)
        gx = ax.ax_matmul_backward(gy.cuda(), x.cuda(), v.cuda(), transposed=t, gw_out=False, gb_out=False)[0]
        want, size = _product(gy.double(), vd.t())
        F.assert_within(gx, want, size * F.sum_bound(N, dt == "f32") + want.abs() * F.store(dtype), "gx")


def test_other_streams():
    """Calls on a stream that is not the current one, their workspaces and results allocated inside."""
    g = F.gen(8)
    x, w, wu = F.randn(g, (257, 320)).cuda(), F.randn(g, (320, 136), 0.05).cuda(), F.randn(g, (320, 136), 0.05).cuda()
    want = ax.ax_gated(x, w, wu, save=True)
    grad = ax.ax_gated_backward(want[0], x, w, wu, want[1], want[2])
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for _ in range(3):
        got = ax.ax_gated(x, w, wu, save=True, stream=s)
        out = ax.ax_gated_backward(got[0], x, w, wu, got[1], got[2], stream=s)
        s.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and all(torch.equal(a, b) for a, b in zip(out, grad))


def test_gradients_inside_wider_buffers():
    g, M, K, N = F.gen(4), 40, 48, 56
    big = torch.full((K, N + 8), 3.0, device="cuda", dtype=torch.bfloat16)
    w = torch.empty_strided((K, N), (N + 8, 1), dtype=torch.bfloat16, device="cuda").copy_(F.randn(g, (K, N)).cuda())
    x, gy = F.randn(g, (M, K), 1.0, torch.bfloat16).cuda(), F.randn(g, (M, N), 1.0, torch.bfloat16).cuda()
    want = ax.ax_matmul_backward(gy, x, w.contiguous())
    ax.ax_matmul_backward(gy, x, w, gw_out=big[:, :N])
    assert torch.equal(big[:, :N], want[1]) and bool((big[:, N:] == 3.0).all())


def test_non_finite_operands_show_where_they_are_used():
    x, w = torch.ones((40, 96)), torch.ones((96, 72))
    x[3, 5], x[7, 9], w[2, 30] = float("nan"), float("inf"), float("-inf")
    for dtype in (torch.float32, torch.bfloat16):
        y, _ = ax.ax_matmul(x.to(dtype).cuda(), w.to(dtype).cuda())
        ok = torch.isfinite(y.float().cpu())
        want = torch.ones((40, 72), dtype=torch.bool)
        want[3], want[7], want[:, 30] = False, False, False
        assert torch.equal(ok, want)


def test_no_rows():
    x, w, gy = torch.empty((0, 24), device="cuda"), torch.ones((24, 40), device="cuda"), torch.empty((0, 40), device="cuda")
    assert ax.ax_matmul(x, w)[0].shape == (0, 40) and ax.ax_gated(x, w, w)[0].shape == (0, 40)
    full = lambda *s: torch.full(s, 7.0, device="cuda")  # noqa: E731
    gx, gw, gb = ax.ax_matmul_backward(gy, x, w, gw_out=full(24, 40), gb_out=full(40))
    assert gx.shape == (0, 24) and not bool(gw.any()) and not bool(gb.any())
    out = ax.ax_gated_backward(gy, x, w, w, gy, gy, gwg_out=full(24, 40), gwu_out=full(24, 40))
    assert not bool(out[1].any()) and not bool(out[2].any())
    c, s = torch.empty((0, 24), dtype=torch.int8, device="cuda"), torch.empty(0, device="cuda")
    wc, ws = torch.ones((40, 24), dtype=torch.int8, device="cuda"), torch.ones(40, device="cuda")
    assert ax.ax_matmul_q8(c, s, wc, ws).shape == (0, 40) and ax.ax_gated_q8(c, s, wc, ws, wc, ws).shape == (0, 40)


def test_more_elements_than_32_bits_count():
    M, K, N = (1 << 20) + 70, 2112, 16
    x = torch.zeros((M, K), dtype=torch.bfloat16, device="cuda")
    x[-70:] = F.randn(F.gen(1), (70, K), 1.0, torch.bfloat16).cuda()
    w = F.randn(F.gen(2), (K, N), 0.02, torch.bfloat16).cuda()
    y, _ = ax.ax_matmul(x, w)
    zd, size = _product(x[-70:].cpu().double(), w.cpu().double())
    F.assert_within(y[-70:], zd, size * F.sum_bound(K) + zd.abs() * F.store(torch.bfloat16))
    assert not bool(y[:-70].any())
    gy = torch.zeros((M, N), dtype=torch.bfloat16, device="cuda")
    gy[-70:] = F.randn(F.gen(3), (70, N), 1.0, torch.bfloat16).cuda()
    gx, gw, _ = ax.ax_matmul_backward(gy, x, w)
    gd, xd = gy[-70:].cpu().double(), x[-70:].cpu().double()
    F.assert_within(gw, xd.t() @ gd, xd.t().abs() @ gd.abs() * F.sum_bound(M) + (xd.t() @ gd).abs() * F.store(torch.bfloat16), "gw")
    want = gd @ w.cpu().double().t()
    F.assert_within(gx[-70:], want, gd.abs() @ w.cpu().double().t().abs() * F.sum_bound(N) + want.abs() * F.store(torch.bfloat16), "gx")
    assert not bool(gx[:-70].any())
