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
    codes = torch.randint(-8, 8, shape, generator=g, dtype=torch.int8)
    scales = ((torch.rand(shape[:-1] + (-(-shape[-1] // group),), generator=g) + 0.1) * shape[-1] ** -0.5 / 4).to(torch.bfloat16)
    return ax.ax_pack_q4(codes.cuda(), scales.cuda(), group=group), values(codes, scales, group)


def _rounded(M, dtype, used=1):
    """Half a unit of a weight, where they are rounded to bf16 for the tiles."""
    return 2.0 ** -8 * 1.01 if dtype == torch.bfloat16 and M > (192 * used if used > 1 else 256) else 0.0


def _check(y, zd, size, K, weight, act, r, dtype, what):
    zb = size * (F.sum_bound(K, dtype == torch.float32) + weight)
    yd = F.act(zd, act)
    bound = zb * F.ACT_LIP + yd.abs() * F.ACT_REL + F.U * zd.abs()
    if r is not None:
        yd = yd + r
        bound = bound + 2 * F.U * (yd.abs() + r.abs())
    F.assert_within(y, yd, bound + yd.abs() * F.store(dtype), what)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", [(1, 1, 1), (1, 4096, 130), (2, 128, 16), (3, 31, 17), (15, 200, 33), (16, 1000, 48), (17, 129, 64), (31, 2049, 5),
                                   (33, 256, 100), (64, 640, 31), (65, 130, 129), (130, 333, 72), (300, 1024, 264), (700, 96, 40)])
def test_matmul(M, K, N, dt, group):
    dtype, g = F.DT[dt], F.gen(M + K + N + group)
    x, b, r = F.randn(g, (M, K), 1.0, dtype), F.randn(g, (N,), 1.0, dtype), F.randn(g, (M, N), 1.0, dtype)
    q, w = _weights(g, (N, K), group)
    zd, size = x.double() @ w.t(), x.double().abs() @ w.abs().t()
    y = ax.ax_matmul_q4(x.cuda(), q)
    _check(y, zd, size, K, _rounded(M, dtype), "none", None, dtype, "plain")
    zd, size = zd + b.double(), size + F.U * (zd.abs() + b.double().abs()) / F.sum_bound(K)
    for i, act in enumerate(ACTS):
        y = ax.ax_matmul_q4(x.cuda(), q, bias=b.cuda(), residual=r.cuda() if i % 2 else None, act=act)
        _check(y, zd, size, K, _rounded(M, dtype), act, r.double() if i % 2 else None, dtype, act)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("M,K,N", [(1, 64, 33), (16, 1000, 48), (20, 300, 17), (50, 256, 80), (100, 200, 130)])
def test_gated(M, K, N, dt, group, act):
    dtype, g = F.DT[dt], F.gen(M + K + N + group)
    x = F.randn(g, (M, K), 1.0, dtype)
    (qg, wg), (qu, wu) = _weights(g, (N, K), group), _weights(g, (N, K), group)
    xd = x.double()
    gd, gs, ud, us = xd @ wg.t(), xd.abs() @ wg.abs().t(), xd @ wu.t(), xd.abs() @ wu.abs().t()
    s = F.sum_bound(K, dt == "f32") + _rounded(M, dtype)
    hd = F.act(gd, act) * ud
    hb = F.ACT_LIP * gs * s * (ud.abs() + us * s) + F.act(gd, act).abs() * us * s + hd.abs() * (F.ACT_REL + 2 * F.U + F.store(dtype))
    F.assert_within(ax.ax_gated_q4(x.cuda(), qg, qu, act=act), hd, hb)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("sizes", [[1], [0, 2, 0, 1], [16, 0, 17, 31], [3, 1, 2, 0, 0, 40], [100, 0, 90], [70, 64, 0, 65, 129]])
def test_experts(sizes, dt, gated):
    dtype, g, E, K, N, group = F.DT[dt], F.gen(sum(sizes)), len(sizes), 200, 72, 64
    R, T = sum(sizes), max(1, sum(sizes) // 2)
    x = F.randn(g, (T, K), 1.0, dtype)
    index = torch.randint(0, T, (R + 2,), generator=g).to(torch.int32)
    index[R:] = -1
    if R > 3:
        index[1] = T
    offsets = torch.tensor([sum(sizes[:e]) for e in range(E + 1)], dtype=torch.int32)
    (q, w), (qu, wu) = _weights(g, (E, N, K), group), _weights(g, (E, N, K), group)
    in_x = (index[:R] >= 0) & (index[:R] < T)
    xd = x.double()[index[:R].long().clamp(0, T - 1)] * in_x[:, None]
    expert = torch.repeat_interleave(torch.arange(E), torch.tensor(sizes))
    z = lambda v, t: torch.einsum("rk,rnk->rn", t, v[expert])  # noqa: E731
    out = torch.full((R + 2, N), 7.0, dtype=dtype, device="cuda")
    s = F.sum_bound(K, dt == "f32") + _rounded(R + 2, dtype, min(E, R + 2))
    gd, gs = z(w, xd), z(w.abs(), xd.abs())
    dev = dict(offsets=offsets.cuda(), tokens=index.cuda())
    if gated:
        ud, us = z(wu, xd), z(wu.abs(), xd.abs())
        ax.ax_gated_q4(x.cuda(), q, qu, act="silu", h_out=out, **dev)
        yd = F.act(gd, "silu") * ud
        bound = F.ACT_LIP * gs * s * (ud.abs() + us * s) + F.act(gd, "silu").abs() * us * s + yd.abs() * (F.ACT_REL + 2 * F.U + F.store(dtype))
    else:
        ax.ax_matmul_q4(x.cuda(), q, y_out=out, **dev)
        yd, bound = gd, gs * s + gd.abs() * F.store(dtype)
    F.assert_within(out[:R], yd, bound)
    assert bool((out[R:] == 7).all())


@pytest.mark.parametrize("M", [5, 200])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("offset,pad", [(0, 8), (1, 6), (3, 2)])
def test_pitches_and_places(M, dt, offset, pad):
    g, K, N, dtype = F.gen(4), 264, 80, F.DT[dt]
    wide = lambda r, c: F.randn(g, (r, c + offset + pad), 1.0, dtype).cuda()  # noqa: E731
    inner = lambda t: t[:, offset:t.shape[1] - pad]  # noqa: E731
    q, _ = _weights(g, (N, K), 128)
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
    q, _ = _weights(g, (40, 64), 32)
    assert ax.ax_matmul_q4(torch.empty((0, 64), device="cuda"), q).shape == (0, 40)
    assert ax.ax_gated_q4(torch.empty((0, 64), device="cuda"), q, q).shape == (0, 40)
    y = ax.ax_matmul_q4(torch.empty((0, 64), device="cuda"), q, tokens=torch.zeros(3, dtype=torch.int32, device="cuda"))
    assert y.shape == (3, 40) and not bool(y.any())


def test_what_lies_behind_a_row_is_not_looked_at():
    """NaN behind the last column of x, in the same buffer, and between its rows."""
    g = F.gen(2)
    q, w = _weights(g, (30, 100), 32)
    for M in (3, 100):
        buf = torch.full((M, 128), float("nan"), device="cuda")
        buf[:, :100] = F.randn(g, (M, 100)).cuda()
        xd = buf[:, :100].cpu().double()
        zd = xd @ w.t()
        F.assert_within(ax.ax_matmul_q4(buf[:, :100], q), zd, (xd.abs() @ w.abs().t()) * F.sum_bound(100, True) + zd.abs() * F.store(torch.float32))


def test_experts_of_one_matrix_take_all_rows_without_offsets():
    g = F.gen(7)
    q, w = _weights(g, (1, 24, 64), 32)
    x = F.randn(g, (9, 64)).cuda()
    o = torch.tensor([2, 7], dtype=torch.int32).cuda()
    y = ax.ax_matmul_q4(x, q)
    z = ax.ax_matmul_q4(x, q, offsets=o, y_out=torch.full((9, 24), 7.0, device="cuda"))
    assert torch.equal(z[2:7], y[2:7]) and bool((z[:2] == 7).all()) and bool((z[7:] == 7).all())
