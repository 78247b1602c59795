"""Weights of 4 bits: quantization and layout bit by bit, products against 64-bit forms at sizes either side of the kernels' tiles."""

import pytest
import torch

import ff_common as F
from paper_2002_09481_amd import binding as ax

pytestmark = pytest.mark.gpu

ACTS = ["none", "relu", "silu", "gelu"]


def plain_quantized(w, group):
    """Codes (int8) and scales (bf16) of [..., K] float weights, each step a float32 operation."""
    K = w.shape[-1]
    n = -(-K // group)
    p = torch.nn.functional.pad(w.float(), (0, n * group - K)).reshape(*w.shape[:-1], n, group)
    scales = (p.abs().amax(dim=-1) / 7.0).to(torch.bfloat16)
    s = scales.float()[..., None]
    codes = torch.where((s > 0) & torch.isfinite(s), torch.round(p / s).clamp(-8, 7), torch.zeros_like(p))
    return codes.reshape(*w.shape[:-1], n * group)[..., :K].to(torch.int8), scales


def values(codes, scales, group):
    return codes.double() * scales.double().repeat_interleave(group, dim=-1)[..., :codes.shape[-1]]


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 1), (16, 128), (17, 129), (3, 40), (100, 1000), (33, 4096), (2, 17, 65), (5, 16, 256), (3, 1, 31)])
def test_quantization(shape, dt, group):
    g = F.gen(sum(shape) + group)
    w = F.randn(g, shape, 0.05, F.DT[dt])
    w[..., -1, :][..., : shape[-1] // 2] = 0.0
    if shape[-2] > 4:
        w[..., 1, :] = 0.0
        w[..., 2, :] *= 2.0 ** -120
    q = ax.ax_quantize_q4(w.cuda(), group=group)
    codes, scales = plain_quantized(w, group)
    want = codes.float() * scales.float().repeat_interleave(group, dim=-1)[..., :shape[-1]]
    got = q.values()
    assert q.shape == shape and got.shape == torch.Size(shape) and torch.equal(got.cpu(), want)
    again = ax.ax_pack_q4(codes.cuda(), scales.cuda(), group=group)
    assert torch.equal(again.codes, q.codes) and torch.equal(again.scales, q.scales)


def test_quantization_of_rows_in_wider_buffers():
    g = F.gen(1)
    w = F.randn(g, (3, 20, 70)).cuda()
    inner = w[..., 3:63]
    a, b = ax.ax_quantize_q4(inner, group=32), ax.ax_quantize_q4(inner.contiguous(), group=32)
    assert torch.equal(a.codes, b.codes) and torch.equal(a.scales, b.scales)
    a, b = ax.ax_quantize_q4(inner[1]), ax.ax_quantize_q4(inner[1].contiguous())
    assert torch.equal(a.codes, b.codes) and torch.equal(a.scales, b.scales)


def test_codes_and_scales_from_elsewhere():
    codes = torch.arange(-8, 8, dtype=torch.int8).repeat(5, 9)[:, :130].contiguous()
    scales = (torch.arange(1, 26).view(5, 5) * 0.5).to(torch.bfloat16)
    q = ax.ax_pack_q4(codes.cuda(), scales.cuda(), group=32)
    assert torch.equal(q.values().cpu().double(), values(codes, scales, 32))
    wild = torch.tensor([[-128, -9, -8, 7, 8, 127]], dtype=torch.int8)
    q = ax.ax_pack_q4(wild.cuda(), torch.ones((1, 1), dtype=torch.bfloat16).cuda())
    assert q.values().cpu().tolist() == [[-8.0, -8.0, -8.0, 7.0, 7.0, 7.0]]


def test_groups_that_are_not_finite():
    w = torch.ones((4, 256))
    w[1, 3], w[2, 200] = float("nan"), float("inf")
    v = ax.ax_quantize_q4(w.cuda()).values().cpu()
    ok = torch.ones((4, 256), dtype=torch.bool)
    ok[1, :128], ok[2, 128:] = False, False
    assert torch.equal(torch.isfinite(v), ok) and bool(((v - 1).abs()[ok] <= 2.0 ** -8).all())


def _weights(g, shape, group):
    """(weights, their values, an absolute bound of what is summed in their place where bf16 rows meet codes with 24 added: those are 31 at
    most, and 24 is taken off again)."""
    codes = torch.randint(-8, 8, shape, generator=g, dtype=torch.int8)
    scales = ((torch.rand(shape[:-1] + (-(-shape[-1] // group),), generator=g) + 0.1) * shape[-1] ** -0.5 / 4).to(torch.bfloat16)
    return ax.ax_pack_q4(codes.cuda(), scales.cuda(), group=group), values(codes, scales, group), values(torch.ones_like(codes), scales, group) * 55


def _way(rows, N, used=1, gated=False, dtype=torch.bfloat16):
    """Which kernel a call takes: few rows, tiles, or weights written out."""
    units = used * -(-rows // (64 * used)) * -(-N // 16) * (2 if gated else 1)
    if rows <= 32 * used or units <= 1024:
        return "few"
    return "written" if dtype == torch.bfloat16 and rows > 600 * used else "tiles"


def _sums(xd, w, most, K, way, dtype):
    """Bound of a product's sum: of its terms, or of what is summed in their place; half a unit of every weight where they are rounded."""
    a = xd.abs()
    size = a @ w.abs().t()
    if way == "tiles" and dtype == torch.bfloat16:
        return (a @ most.t()) * F.sum_bound(K)
    return size * (F.sum_bound(K, dtype == torch.float32) + (2.0 ** -8 * 1.01 if way == "written" else 0))


def _check(y, zd, zb, act, r, dtype, what):
    yd = F.act(zd, act)
    bound = zb * F.ACT_LIP + yd.abs() * F.ACT_REL + F.U * zd.abs()
    if r is not None:
        yd = yd + r
        bound = bound + 2 * F.U * (yd.abs() + r.abs())
    F.assert_within(y, yd, bound + yd.abs() * F.store(dtype), what)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N,way", [(1, 1, 1, "few"), (1, 4096, 130, "few"), (2, 128, 16, "few"), (3, 31, 17, "few"), (15, 200, 33, "few"),
                                       (16, 1000, 48, "few"), (17, 129, 64, "few"), (31, 2049, 5, "few"), (33, 256, 100, "few"), (64, 640, 31, "few"),
                                       (65, 130, 129, "few"), (130, 333, 72, "few"), (300, 1024, 264, "few"), (700, 96, 40, "few"), (8, 64, 9000, "few"),
                                       (70, 65, 8300, "tiles"), (33, 1, 16400, "tiles"), (129, 130, 6000, "tiles"), (300, 520, 3601, "tiles"),
                                       (600, 63, 1700, "tiles"), (601, 31, 1650, None), (650, 264, 1601, None)])
def test_matmul(M, K, N, way, dt, group):
    dtype, g = F.DT[dt], F.gen(M + K + N + group)
    assert way in (None, _way(M, N, dtype=dtype))
    way = _way(M, N, dtype=dtype)
    x, b, r = F.randn(g, (M, K), 1.0, dtype), F.randn(g, (N,), 1.0, dtype), F.randn(g, (M, N), 1.0, dtype)
    q, w, most = _weights(g, (N, K), group)
    xd = x.double()
    zd, zb = xd @ w.t(), _sums(xd, w, most, K, way, dtype)
    y = ax.ax_matmul_q4(x.cuda(), q)
    _check(y, zd, zb, "none", None, dtype, "plain")
    zd = zd + b.double()
    zb = zb + F.U * (zd.abs() + b.double().abs())
    for i, act in enumerate(ACTS):
        y = ax.ax_matmul_q4(x.cuda(), q, bias=b.cuda(), residual=r.cuda() if i % 2 else None, act=act)
        _check(y, zd, zb, act, r.double() if i % 2 else None, dtype, act)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", [(1, 64, 33), (16, 1000, 48), (20, 300, 17), (50, 256, 80), (100, 200, 130), (300, 200, 1901), (40, 129, 8200), (700, 96, 903)])
def test_gated(M, K, N, dt, group, act):
    dtype, g = F.DT[dt], F.gen(M + K + N + group)
    x = F.randn(g, (M, K), 1.0, dtype)
    (qg, wg, mg), (qu, wu, mu) = _weights(g, (N, K), group), _weights(g, (N, K), group)
    xd, way = x.double(), _way(M, N, gated=True, dtype=dtype)
    gd, ud, gb, ub = xd @ wg.t(), xd @ wu.t(), _sums(xd, wg, mg, K, way, dtype), _sums(xd, wu, mu, K, way, dtype)
    hd = F.act(gd, act) * ud
    hb = F.ACT_LIP * gb * (ud.abs() + ub) + F.act(gd, act).abs() * ub + hd.abs() * (F.ACT_REL + 2 * F.U + F.store(dtype))
    F.assert_within(ax.ax_gated_q4(x.cuda(), qg, qu, act=act), hd, hb)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("sizes,K,N", [([1], 200, 72), ([0, 2, 0, 1], 200, 72), ([16, 0, 17, 31], 200, 72), ([3, 1, 2, 0, 0, 40], 200, 72),
                                       ([100, 0, 90], 200, 72), ([70, 64, 0, 65, 129], 200, 2101), ([300, 0, 513, 2, 400], 136, 2100), ([0, 0, 777], 65, 1000),
                                       ([1500, 2, 1100], 64, 400), ([40, 31, 0, 64, 33, 1], 72, 4096)])
def test_experts(sizes, K, N, dt, gated):
    dtype, g, E, group = F.DT[dt], F.gen(sum(sizes)), len(sizes), 64
    R, T = sum(sizes), max(1, sum(sizes) // 2)
    x = F.randn(g, (T, K), 1.0, dtype)
    index = torch.randint(0, T, (R + 2,), generator=g).to(torch.int32)
    index[R:] = -1
    if R > 3:
        index[1] = T
    offsets = torch.tensor([sum(sizes[:e]) for e in range(E + 1)], dtype=torch.int32)
    (q, w, most), (qu, wu, mostu) = _weights(g, (E, N, K), group), _weights(g, (E, N, K), group)
    in_x = (index[:R] >= 0) & (index[:R] < T)
    xd = x.double()[index[:R].long().clamp(0, T - 1)] * in_x[:, None]
    way = _way(R + 2, N, min(E, R + 2), gated, dtype)
    parts = lambda v, m: [torch.cat(t) for t in zip(*[(p @ v[e].t(), _sums(p, v[e], m[e], K, way, dtype)) for e, p in enumerate(xd.split(sizes))])]  # noqa: E731
    out = torch.full((R + 2, N), 7.0, dtype=dtype, device="cuda")
    gd, gb = parts(w, most)
    dev = dict(offsets=offsets.cuda(), tokens=index.cuda())
    if gated:
        ud, ub = parts(wu, mostu)
        ax.ax_gated_q4(x.cuda(), q, qu, act="silu", h_out=out, **dev)
        yd = F.act(gd, "silu") * ud
        bound = F.ACT_LIP * gb * (ud.abs() + ub) + F.act(gd, "silu").abs() * ub + yd.abs() * (F.ACT_REL + 2 * F.U + F.store(dtype))
    else:
        ax.ax_matmul_q4(x.cuda(), q, y_out=out, **dev)
        yd, bound = gd, gb + gd.abs() * F.store(dtype)
    F.assert_within(out[:R], yd, bound)
    assert bool((out[R:] == 7).all())


@pytest.mark.parametrize("M,N", [(5, 80), (500, 2100), (700, 1600)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("offset,pad", [(0, 8), (1, 6), (3, 2)])
def test_pitches_and_places(M, N, dt, offset, pad):
    g, K, dtype = F.gen(4), 264, F.DT[dt]
    wide = lambda r, c: F.randn(g, (r, c + offset + pad), 1.0, dtype).cuda()  # noqa: E731
    inner = lambda t: t[:, offset:t.shape[1] - pad]  # noqa: E731
    q, _, _ = _weights(g, (N, K), 128)
    x, r, buf = inner(wide(M, K)), inner(wide(M, N)), wide(M, N)
    old = buf.clone()
    want = ax.ax_matmul_q4(x.contiguous(), q, residual=r.contiguous(), act="silu")
    ax.ax_matmul_q4(x, q, residual=r, act="silu", y_out=inner(buf))
    assert torch.equal(inner(buf), want)
    inner(buf)[:] = inner(old)
    assert torch.equal(buf, old)
    assert torch.equal(ax.ax_gated_q4(x, q, q), ax.ax_gated_q4(x.contiguous(), q, q))
    rc = r.contiguous()
    assert ax.ax_matmul_q4(x, q, residual=rc, act="silu", y_out=rc) is rc and torch.equal(rc, want)


def test_no_rows_and_no_x():
    g = F.gen(0)
    q, _, _ = _weights(g, (40, 64), 32)
    assert ax.ax_matmul_q4(torch.empty((0, 64), device="cuda"), q).shape == (0, 40)
    assert ax.ax_gated_q4(torch.empty((0, 64), device="cuda"), q, q).shape == (0, 40)
    y = ax.ax_matmul_q4(torch.empty((0, 64), device="cuda"), q, tokens=torch.zeros(3, dtype=torch.int32, device="cuda"))
    assert y.shape == (3, 40) and not bool(y.any())


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows,N", [(3, 40), (300, 3700), (700, 1650)])
def test_rows_of_an_empty_x(rows, N, dt):
    """Every index lies outside: rows of zeros, whichever kernel."""
    q, _, _ = _weights(F.gen(1), (N, 264), 64)
    x, t = torch.empty((0, 264), dtype=F.DT[dt], device="cuda"), torch.arange(-1, rows - 1, dtype=torch.int32, device="cuda")
    b = torch.ones(N, dtype=F.DT[dt], device="cuda")
    assert bool((ax.ax_matmul_q4(x, q, bias=b, tokens=t) == 1).all()) and not bool(ax.ax_gated_q4(x, q, q, tokens=t).any())


def test_what_lies_behind_a_row_is_not_looked_at():
    """NaN behind the last column of x, in the same buffer, and between its rows."""
    g = F.gen(2)
    for M, N in ((3, 30), (300, 3700), (700, 1650)):
        q, w, most = _weights(g, (N, 100), 32)
        for dtype in (torch.float32, torch.bfloat16):
            for cols in (100, 104):  # (of the buffer: rows of whole 16 bytes or not)
                buf = torch.full((M, cols + 28), float("nan"), device="cuda", dtype=dtype)
                buf[:, :100] = F.randn(g, (M, 100), 1.0, dtype).cuda()
                xd = buf[:, :100].cpu().double()
                zd = xd @ w.t()
                F.assert_within(ax.ax_matmul_q4(buf[:, :100], q), zd, _sums(xd, w, most, 100, _way(M, N, dtype=dtype), dtype) + zd.abs() * F.store(dtype))


def test_experts_of_one_matrix_take_all_rows_without_offsets():
    g = F.gen(7)
    q, _, _ = _weights(g, (1, 24, 64), 32)
    x = F.randn(g, (9, 64)).cuda()
    o = torch.tensor([2, 7], dtype=torch.int32).cuda()
    y = ax.ax_matmul_q4(x, q)
    z = ax.ax_matmul_q4(x, q, offsets=o, y_out=torch.full((9, 24), 7.0, device="cuda"))
    assert torch.equal(z[2:7], y[2:7]) and bool((z[:2] == 7).all()) and bool((z[7:] == 7).all())
