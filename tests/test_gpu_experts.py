"""Products of rows grouped by expert and their gradients against 64-bit forms: ragged and empty experts, indexed rows, rows that
belong to nobody, sizes either side of the kernels' tiles, pitches, streams, offsets that make no sense."""

import pytest
import torch

import ff_common as F
from paper_2002_09481_amd import binding as ax

pytestmark = pytest.mark.gpu

ACTS = ["none", "relu", "silu", "gelu"]
# experts' sizes, K, N: few rows each and many, experts without rows at the ends and in the middle, tiles' edges
SIZES = [([1], 1, 1), ([0, 3, 0, 1], 64, 48), ([2, 1, 0, 5, 1, 0, 0], 1000, 33), ([16, 0, 17, 31], 520, 264), ([40, 1, 33], 72, 130),
         ([130, 0, 257, 64, 5], 136, 264), ([300], 200, 129), ([0, 0, 700], 256, 256), ([65, 64, 63, 129, 0, 128, 127], 96, 512)]


def _case(sizes, K, N, dtype, g, transposed=False, weights=1, tokens=None):
    """Rows of x found through an index (with repeats), and some rows at the end that belong to nobody."""
    R, E = sum(sizes), len(sizes)
    T = tokens or max(1, (R * 2) // 3)
    x = F.randn(g, (T, K), 1.0, dtype)
    index = torch.randint(0, T, (R + 3,), generator=g).to(torch.int32)
    index[R:] = -1
    offsets = torch.tensor([sum(sizes[:e]) for e in range(E + 1)], dtype=torch.int32)
    shape = (E, N, K) if transposed else (E, K, N)
    ws = [F.randn(g, shape, K ** -0.5, dtype) for _ in range(weights)]
    expert = torch.repeat_interleave(torch.arange(E), torch.tensor(sizes))
    return x, index, offsets, ws, expert, R


def _grouped(x, w, expert, transposed=False):
    """Rows of x (64 bits) times the matrix of their expert, and the absolute sum of its terms."""
    N = w.shape[1] if transposed else w.shape[2]
    z, size = torch.zeros((x.shape[0], N), dtype=torch.float64), torch.zeros((x.shape[0], N), dtype=torch.float64)
    for e in range(w.shape[0]):
        at = expert == e
        m = w[e].double().t() if transposed else w[e].double()
        z[at], size[at] = x[at] @ m, x[at].abs() @ m.abs()
    return z, size


def _summed(x, gz, bound, expert, E):
    """x^T gz of every expert's rows, the sum of |x|^T bound and of |x|^T |gz|."""
    out = [torch.zeros((E, x.shape[1], gz.shape[1]), dtype=torch.float64) for _ in range(3)]
    for e in range(E):
        at = expert == e
        out[0][e], out[1][e], out[2][e] = x[at].t() @ gz[at], x[at].abs().t() @ bound[at], x[at].abs().t() @ gz[at].abs()
    return out


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("case", range(len(SIZES)))
def test_matmul(case, dt, transposed):
    sizes, K, N = SIZES[case]
    dtype, g, f32 = F.DT[dt], F.gen(case), dt == "f32"
    x, index, offsets, (w,), expert, R = _case(sizes, K, N, dtype, g, transposed)
    xd = x.double()[index[:R].long()]
    zd, size = _grouped(xd, w, expert, transposed)
    dev = [t.cuda() for t in (x, w, offsets, index)]
    for act in ACTS:
        mark = lambda: torch.full((R + 3, N), 7.0, dtype=dtype, device="cuda")  # noqa: E731
        y, z = ax.ax_matmul_experts(*dev, act=act, transposed=transposed, y_out=mark(), z_out=mark())
        zb = size * F.sum_bound(K, f32)
        F.assert_within(z[:R], zd, zb + zd.abs() * F.store(dtype), act + " z")
        yd = F.act(zd, act)
        F.assert_within(y[:R], yd, zb * F.ACT_LIP + yd.abs() * (F.ACT_REL + F.store(dtype)), act + " y")
        assert bool((y[R:] == 7).all()) and bool((z[R:] == 7).all())
    # the rows themselves, without an index
    rows = x[index.long()].cuda()  # (as many of them: their number decides the kernel)
    again, none = ax.ax_matmul_experts(rows, dev[1], dev[2], act=act, transposed=transposed)
    assert none is None and torch.equal(again[:R], y[:R])


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("act", ["none", "gelu"])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("case", range(len(SIZES)))
def test_matmul_gradients(case, dt, act, transposed):
    sizes, K, N = SIZES[case]
    dtype, g, f32, E = F.DT[dt], F.gen(100 + case), dt == "f32", len(SIZES[case][0])
    x, index, offsets, (w,), expert, R = _case(sizes, K, N, dtype, g, transposed)
    xd = x.double()[index[:R].long()]
    gy, z = F.randn(g, (R + 3, N), 1.0, dtype), F.randn(g, (R + 3, N), 1.0, dtype)
    gy[R:] = float("nan")  # (rows of nobody)
    gz = gy[:R].double() * (F.slope(z[:R].double(), act) if act != "none" else 1)
    one = (24 * F.U * gy[:R].double().abs() if act != "none" else 0 * gz.abs()) + (gz.abs() * 2.0 ** -8 if act != "none" and not f32 else 0)
    dev = [t.cuda() for t in (gy, x, w, offsets, index)]
    kw = dict(z=z.cuda() if act != "none" else None, act=act, transposed=transposed)
    gx, gw = ax.ax_matmul_experts_backward(*dev, gx_out=torch.full((R + 3, K), 7.0, dtype=dtype, device="cuda"), **kw)
    want, size = _grouped(gz, w, expert, not transposed)
    bound, _ = _grouped(one, w.abs(), expert, not transposed)
    F.assert_within(gx[:R], want, bound + size * F.sum_bound(N, f32) + want.abs() * F.store(dtype), "gx")
    assert bool((gx[R:] == 7).all())
    want, bound, size = _summed(xd, gz, one, expert, E)
    bound = bound + size * F.sum_bound(max(sizes), f32) + want.abs() * F.store(dtype)
    if transposed:
        want, bound = want.transpose(1, 2), bound.transpose(1, 2)
    F.assert_within(gw, want, bound, "gw")
    only = ax.ax_matmul_experts_backward(*dev, gw_out=False, **kw)
    assert only[1] is None and torch.equal(only[0][:R], gx[:R])
    only = ax.ax_matmul_experts_backward(*dev, gx_out=False, **kw)
    assert only[0] is None and torch.equal(only[1], gw)
    again = ax.ax_matmul_experts_backward(dev[0], x[index.long()].cuda(), *dev[2:4], **kw)
    assert torch.equal(again[0][:R], gx[:R]) and torch.equal(again[1], gw)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("case", range(len(SIZES)))
def test_gated(case, dt, act):
    sizes, K, N = SIZES[case]
    dtype, g, f32, E = F.DT[dt], F.gen(200 + case), dt == "f32", len(SIZES[case][0])
    x, index, offsets, (wg, wu), expert, R = _case(sizes, K, N, dtype, g, weights=2)
    xd = x.double()[index[:R].long()]
    dev = [t.cuda() for t in (x, wg, wu, offsets, index)]
    h, gp, up = ax.ax_gated_experts(*dev, act=act, save=True)
    (gd, gs), (ud, us), s = _grouped(xd, wg, expert), _grouped(xd, wu, expert), F.sum_bound(K, f32)
    F.assert_within(gp[:R], gd, gs * s + gd.abs() * F.store(dtype), "g")
    F.assert_within(up[:R], ud, us * s + ud.abs() * F.store(dtype), "u")
    hd = F.act(gd, act) * ud
    hb = F.ACT_LIP * gs * s * (ud.abs() + us * s) + F.act(gd, act).abs() * us * s + hd.abs() * (F.ACT_REL + 2 * F.U + F.store(dtype))
    F.assert_within(h[:R], hd, hb, "h")
    assert torch.equal(h[:R], ax.ax_gated_experts(*dev, act=act)[0][:R])

    gh, gv, uv = (F.randn(g, (R + 3, N), 1.0, dtype) for _ in range(3))
    out = ax.ax_gated_experts_backward(gh.cuda(), *dev[:3], gv.cuda(), uv.cuda(), *dev[3:], act=act)
    gh, gv, uv = (t[:R].double() for t in (gh, gv, uv))
    gg, gu = gh * uv * F.slope(gv, act), gh * F.act(gv, act)
    low = 0 if f32 else 2.0 ** -8
    bg, bu = 24 * F.U * (gh * uv).abs() + gg.abs() * low, 24 * F.U * (gh * gv).abs() + gu.abs() * low
    (a, sa), (b, sb) = _grouped(gg, wg, expert, True), _grouped(gu, wu, expert, True)
    bound = _grouped(bg, wg.abs(), expert, True)[0] + _grouped(bu, wu.abs(), expert, True)[0]
    F.assert_within(out[0][:R], a + b, bound + (sa + sb) * F.sum_bound(2 * N, f32) + (a + b).abs() * F.store(dtype), "gx")
    for o, v, bv, n in ((out[1], gg, bg, "gwg"), (out[2], gu, bu, "gwu")):
        want, bound, size = _summed(xd, v, bv, expert, E)
        F.assert_within(o, want, bound + size * F.sum_bound(max(sizes), f32) + want.abs() * F.store(dtype), n)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("R,E", [(4, 3), (200, 3)])
@pytest.mark.parametrize("offset,pad", [(0, 16), (1, 6), (5, 11)])
def test_pitches_and_places(dt, R, E, offset, pad):
    """Operands and outputs inside wider buffers, at any element: the bits of the contiguous call, nothing else written."""
    g, K, N, dtype = F.gen(4), 144, 208, F.DT[dt]
    wide = lambda *s: F.randn(g, s[:-1] + (s[-1] + offset + pad,), 1.0, dtype).cuda()  # noqa: E731
    inner = lambda t: t[..., offset:t.shape[-1] - pad]  # noqa: E731
    x, w, w2, gy = inner(wide(R, K)), inner(wide(E, K, N)), inner(wide(E, K, N)), inner(wide(R, N))
    o = torch.tensor([0, R // 2, R // 2, R], dtype=torch.int32).cuda()
    t = torch.randperm(R, generator=g).to(torch.int32).cuda()
    c = lambda *a: [v.contiguous() for v in a]  # noqa: E731
    buf = wide(R, N)
    old = buf.clone()
    for tokens in (None, t):
        ref, z = ax.ax_matmul_experts(*c(x, w), o, tokens, act="silu", save=True)
        ax.ax_matmul_experts(x, w, o, tokens, act="silu", y_out=inner(buf))
        assert torch.equal(inner(buf), ref)
        inner(buf)[:] = inner(old)
        assert torch.equal(buf, old)
        gw = inner(wide(E, K, N))
        out = ax.ax_matmul_experts_backward(gy, x, w, o, tokens, z=z, act="silu", gw_out=gw, gx_out=inner(wide(R, K)))
        assert all(torch.equal(a, b) for a, b in zip(out, ax.ax_matmul_experts_backward(*c(gy, x, w), o, tokens, z=z, act="silu")))
        out = ax.ax_matmul_experts_backward(gy, x, w, o, tokens)
        assert all(torch.equal(a, b) for a, b in zip(out, ax.ax_matmul_experts_backward(*c(gy, x, w), o, tokens)))
        assert out[1].stride() == w.stride()
        assert torch.equal(ax.ax_gated_experts(x, w, w2, o, tokens)[0], ax.ax_gated_experts(*c(x, w, w2), o, tokens)[0])
        out = ax.ax_gated_experts_backward(gy, x, w, w2, z, z, o, tokens)
        assert all(torch.equal(a, b) for a, b in zip(out, ax.ax_gated_experts_backward(*c(gy, x, w, w2), z, z, o, tokens)))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("R", [6, 150])
def test_indexes_outside_x_are_rows_of_zeros(R, dt):
    g, dtype, K, N = F.gen(R), F.DT[dt], 96, 72
    x, w = F.randn(g, (5, K), 1.0, dtype).cuda(), F.randn(g, (2, K, N), 1.0, dtype).cuda()
    o = torch.tensor([0, R // 3, R], dtype=torch.int32).cuda()
    t = torch.randint(0, 5, (R,), generator=g).to(torch.int32)
    t[1], t[3], t[R - 1] = -1, 5, 2 ** 31 - 1
    y, _ = ax.ax_matmul_experts(x, w, o, t.cuda())
    out = [i for i in range(R) if not 0 <= int(t[i]) < 5]
    assert not bool(y[out].any())
    full = torch.where((t >= 0) & (t < 5), t, torch.zeros_like(t))
    rows = x[full.long().cuda()]
    rows[out] = 0
    assert torch.equal(y, ax.ax_matmul_experts(rows, w, o)[0])
    gy = F.randn(g, (R, N), 1.0, dtype).cuda()
    assert torch.equal(ax.ax_matmul_experts_backward(gy, x, w, o, t.cuda())[1], ax.ax_matmul_experts_backward(gy, rows, w, o)[1])


@pytest.mark.parametrize("R", [6, 300])
def test_offsets_that_make_no_sense_stay_inside(R):
    """Descending, negative and too large offsets: nothing outside the arrays is written."""
    g, K, N = F.gen(R), 64, 40
    x, w = F.randn(g, (R, K)).cuda(), F.randn(g, (4, K, N)).cuda()
    for bad in ([-7, R // 2, 1, R // 3, 2 ** 31 - 1], [2 ** 31 - 1, -2 ** 31, 0, R, R + 64], [R, R, 0, 0, -1]):
        o = torch.tensor(bad, dtype=torch.int32).cuda()
        buf, gbuf = torch.full((R + 600, N), 7.0, device="cuda"), torch.full((6, K, N), 7.0, device="cuda")
        y, _ = ax.ax_matmul_experts(x, w, o, y_out=buf[300:300 + R])
        assert bool((buf[:300] == 7).all()) and bool((buf[300 + R:] == 7).all()) and bool(torch.isfinite(y).all())
        ax.ax_matmul_experts_backward(torch.ones((R, N), device="cuda"), x, w, o, gw_out=gbuf[1:5])
        assert bool((gbuf[0] == 7).all()) and bool((gbuf[5] == 7).all()) and bool(torch.isfinite(gbuf).all())
    gap = torch.tensor([2, 3, 3, 5, 5], dtype=torch.int32).cuda()  # rows in front of the first and behind the last
    y, _ = ax.ax_matmul_experts(x, w, gap, y_out=torch.full((R, N), 7.0, device="cuda"))
    assert bool((y[:2] == 7).all()) and bool((y[5:] == 7).all()) and not bool((y[2:5] == 7).any())


def test_no_rows():
    x, w, o = torch.empty((0, 24), device="cuda"), torch.ones((2, 24, 40), device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    t = torch.empty(0, dtype=torch.int32, device="cuda")
    full = lambda: torch.full((2, 24, 40), 7.0, device="cuda")  # noqa: E731
    for tokens in (None, t):
        assert ax.ax_matmul_experts(x, w, o, tokens)[0].shape == (0, 40) and ax.ax_gated_experts(x, w, w, o, tokens)[0].shape == (0, 40)
        gy = torch.empty((0, 40), device="cuda")
        gx, gw = ax.ax_matmul_experts_backward(gy, x, w, o, tokens, gw_out=full())
        assert gx.shape == (0, 24) and not bool(gw.any())
        out = ax.ax_gated_experts_backward(gy, x, w, w, gy, gy, o, tokens, gwg_out=full(), gwu_out=full())
        assert not bool(out[1].any()) and not bool(out[2].any())
    # rows, but none that belong to an expert
    x = torch.ones((50, 24), device="cuda")
    y, _ = ax.ax_matmul_experts(x, w, o, y_out=torch.full((50, 40), 7.0, device="cuda"))
    assert bool((y == 7).all())
    assert not bool(ax.ax_matmul_experts_backward(y, x, w, o, gw_out=full())[1].any())


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [3, 700])
def test_rows_of_an_empty_x(rows, dt):
    """Every index lies outside: rows of zeros."""
    K, N, kw = 264, 520, dict(dtype=F.DT[dt], device="cuda")
    x, w, gy = torch.empty((0, K), **kw), torch.ones((2, K, N), **kw), torch.ones((rows, N), **kw)
    o, t = torch.tensor([0, 1, rows], dtype=torch.int32).cuda(), torch.arange(-1, rows - 1, dtype=torch.int32, device="cuda")
    for transposed in (False, True):
        v = w.transpose(1, 2).contiguous() if transposed else w
        y, z = ax.ax_matmul_experts(x, v, o, t, transposed=transposed, save=True)
        assert y.shape == (rows, N) and not bool(y.any()) and not bool(z.any())
        gx, gw = ax.ax_matmul_experts_backward(gy, x, v, o, t, transposed=transposed, gw_out=torch.ones_like(v))
        assert bool((gx == N).all()) and not bool(gw.any())
    assert not any(bool(v.any()) for v in ax.ax_gated_experts(x, w, w, o, t, save=True))


def test_many_experts():
    """More than a wave looks up at a time."""
    g, E, K, N = F.gen(11), 1024, 16, 24
    for most in (2, 40):
        sizes = torch.randint(0, most, (E,), generator=g).tolist()
        x, index, offsets, (w,), expert, R = _case(sizes, K, N, torch.float32, g)
        zd, size = _grouped(x.double()[index[:R].long()], w, expert)
        y, _ = ax.ax_matmul_experts(x.cuda(), w.cuda(), offsets.cuda(), index.cuda())
        F.assert_within(y[:R], zd, size * F.sum_bound(K, True) + zd.abs() * F.store(torch.float32))
        gy = F.randn(g, (R + 3, N))
        gw = ax.ax_matmul_experts_backward(gy.cuda(), x.cuda(), w.cuda(), offsets.cuda(), index.cuda())[1]
        want, _, size = _summed(x.double()[index[:R].long()], gy[:R].double(), gy[:R].double().abs(), expert, E)
        F.assert_within(gw, want, size * F.sum_bound(most, True) + want.abs() * F.store(torch.float32))


def test_gradients_against_differences():
    """A loss of both products along one direction of all their inputs: central differences of the 64-bit form."""
    g, sizes, K, N = F.gen(21), [2, 0, 4], 20, 12
    x, index, offsets, (wg, wu), expert, R = _case(sizes, K, N, torch.float32, g, weights=2)
    wd, c = F.randn(g, (3, N, K)), F.randn(g, (R, K))
    index = index[:R]
    d = [F.randn(g, t.shape).double() for t in (x, wg, wu, wd)]

    def loss(e):
        X, G, U_, D = (t.double() + e * v for t, v in zip((x, wg, wu, wd), d))
        X = X[index.long()]
        h = F.act(_grouped(X, G, expert)[0], "silu") * _grouped(X, U_, expert)[0]
        return float((c.double() * F.act(_grouped(h, D, expert)[0], "gelu")).sum())

    X, G, U_, D, C, o, t = (v.cuda() for v in (x, wg, wu, wd, c, offsets, index))
    h, gp, up = ax.ax_gated_experts(X, G, U_, o, t, save=True)
    _, z = ax.ax_matmul_experts(h, D, o, act="gelu", save=True)
    gh, gd = ax.ax_matmul_experts_backward(C, h, D, o, z=z, act="gelu")
    gr, gg, gu = ax.ax_gated_experts_backward(gh, X, G, U_, gp, up, o, t)
    gx = torch.zeros(x.shape).index_add_(0, index.long(), gr.cpu())
    terms = [(a.cpu().double() * v) for a, v in zip((gx, gg, gu, gd), d)]
    got, size = sum(float(v.sum()) for v in terms), sum(float(v.abs().sum()) for v in terms)
    e = 1e-5
    slope = (loss(e) - loss(-e)) / (2 * e)
    third = abs(loss(1e-2) - 2 * loss(5e-3) + 2 * loss(-5e-3) - loss(-1e-2)) / (2 * 5e-3 ** 3)
    assert abs(got - slope) <= e * e * third + 1e-15 * size / e + size * 200 * F.U


def test_non_finite_operands_show_in_their_rows_alone():
    for R in (8, 80):
        x, w = torch.ones((R, 96)), torch.ones((2, 96, 72))
        x[3, 5], w[1, 2, 30] = float("nan"), float("inf")
        o = torch.tensor([0, R // 2, R], dtype=torch.int32).cuda()
        for dtype in (torch.float32, torch.bfloat16):
            ok = torch.isfinite(ax.ax_matmul_experts(x.to(dtype).cuda(), w.to(dtype).cuda(), o)[0].float().cpu())
            want = torch.ones((R, 72), dtype=torch.bool)
            want[3], want[R // 2:, 30] = False, False
            assert torch.equal(ok, want)


def test_more_elements_than_32_bits_count():
    """Rows of x, of the products and of a sum beyond 2^31 elements."""
    T, K, N, dtype = (1 << 20) + 70, 2112, 16, torch.bfloat16
    x = torch.zeros((T, K), dtype=dtype, device="cuda")
    x[-70:] = F.randn(F.gen(1), (70, K), 1.0, dtype).cuda()
    w = F.randn(F.gen(2), (2, K, N), 0.02, dtype).cuda()
    xd, wd = x[-70:].cpu().double(), w.cpu().double()
    # few rows and many, found at the end of x
    for R in (20, 70):
        index = torch.arange(T - R, T, dtype=torch.int32).cuda()
        o = torch.tensor([0, 5, R], dtype=torch.int32).cuda()
        y, _ = ax.ax_matmul_experts(x, w, o, index)
        want, size = _grouped(xd[70 - R:], w.cpu(), torch.tensor([0] * 5 + [1] * (R - 5)))
        F.assert_within(y, want, size * F.sum_bound(K) + want.abs() * F.store(dtype))
    # all rows: the last expert's at the end
    o = torch.tensor([0, T - 70, T], dtype=torch.int32).cuda()
    y, _ = ax.ax_matmul_experts(x, w, o)
    want = xd @ wd[1]
    F.assert_within(y[-70:], want, (xd.abs() @ wd[1].abs()) * F.sum_bound(K) + want.abs() * F.store(dtype))
    assert not bool(y[:-70].any())
    gy = F.randn(F.gen(3), (T, N), 1.0, dtype).cuda()
    gx, gw = ax.ax_matmul_experts_backward(gy, x, w, o)
    gd = gy[-70:].cpu().double()
    want = gd @ wd[1].t()
    F.assert_within(gx[-70:], want, (gd.abs() @ wd[1].t().abs()) * F.sum_bound(N) + want.abs() * F.store(dtype), "gx")
    want = xd.t() @ gd
    F.assert_within(gw[1], want, (xd.t().abs() @ gd.abs()) * F.sum_bound(70) + want.abs() * F.store(dtype), "gw")
    assert not bool(gw[0].any())
    rows = torch.tensor([[T - 1, 0], [T - 3, T - 1]], dtype=torch.int32).cuda()
    assert torch.equal(ax.ax_combine(x, rows), torch.stack((x[-1], (x[-3].float() + x[-1].float()).to(dtype))))
    two = x[-2:].clone()
    gh, gr = ax.ax_combine_backward(two, x, rows[:, :1].contiguous())
    assert torch.equal(gh[T - 1], two[0]) and torch.equal(gh[T - 3], two[1])
    want = torch.stack((two[0].double() @ x[-1].double(), two[1].double() @ x[-3].double()))[:, None].cpu()
    size = torch.stack((two[0].double().abs() @ x[-1].double().abs(), two[1].double().abs() @ x[-3].double().abs()))[:, None].cpu()
    F.assert_within(gr, want, size * (K / 64 + 24) * 2 * F.U)
