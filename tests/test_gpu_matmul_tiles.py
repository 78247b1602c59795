"""Every tile of the matrix products, in one piece and with a contraction in slices, in every layout and type of result.

The sizes are odd and as small as the choice of tile allows; the test asks for that choice, so that a size whose tile changes is
noticed and replaced.  References are 64-bit products."""

import pytest
import torch

import ff_common as F
from paper_2002_09481_amd import binding as ax

pytestmark = pytest.mark.gpu

# (product, type, transposed, M, K, N, rows of the tile, in slices)
CASES = [
    ("matmul", "bf16", False, 33, 40, 129, 32, False), ("matmul", "bf16", False, 33, 1000, 129, 32, True),
    ("matmul", "bf16", False, 8197, 40, 129, 64, False), ("matmul", "bf16", False, 2051, 4104, 129, 64, True),
    ("matmul", "bf16", False, 641, 40, 6003, 128, False), ("matmul", "bf16", False, 4101, 4104, 129, 128, True),
    ("matmul", "bf16", False, 8197, 40, 1003, 256, False), ("matmul", "bf16", True, 33, 40, 129, 32, False),
    ("matmul", "bf16", True, 33, 1000, 129, 32, True), ("matmul", "bf16", True, 8197, 40, 129, 64, False),
    ("matmul", "bf16", True, 2051, 4104, 129, 64, True), ("matmul", "bf16", True, 641, 40, 6003, 128, False),
    ("matmul", "bf16", True, 4101, 4104, 129, 128, True), ("matmul", "bf16", True, 8197, 40, 1003, 256, False),
    ("matmul", "f32", False, 65, 40, 129, 64, False), ("matmul", "f32", False, 65, 520, 129, 64, True),
    ("matmul", "f32", True, 65, 40, 129, 64, False), ("matmul", "f32", True, 65, 520, 129, 64, True),
    ("matmul", "f32", True, 8197, 136, 129, 128, False), ("matmul", "f32", True, 3001, 2050, 129, 128, True),
    ("matmul_q8", "bf16", False, 33, 40, 129, 32, False), ("matmul_q8", "bf16", False, 33, 2050, 129, 32, True),
    ("matmul_q8", "bf16", False, 8197, 40, 129, 64, False), ("matmul_q8", "bf16", False, 641, 40, 6003, 128, False),
    ("matmul_q8", "bf16", False, 8197, 4104, 129, 128, True), ("matmul_q8", "bf16", False, 8197, 40, 1003, 256, False),
    ("gated", "bf16", False, 33, 40, 129, 32, False), ("gated", "bf16", False, 33, 1000, 129, 32, True),
    ("gated", "bf16", False, 6007, 40, 129, 64, False), ("gated", "bf16", False, 33, 4104, 4100, 64, True),
    ("gated", "bf16", False, 333, 40, 6003, 128, False), ("gated", "bf16", False, 65, 4104, 6003, 128, True),
    ("gated", "bf16", False, 641, 40, 6003, 256, False), ("gated", "f32", False, 65, 40, 129, 64, False),
    ("gated", "f32", False, 65, 520, 129, 64, True), ("gated_q8", "bf16", False, 33, 40, 129, 32, False),
    ("gated_q8", "bf16", False, 33, 2050, 129, 32, True), ("gated_q8", "bf16", False, 6007, 40, 129, 64, False),
    ("gated_q8", "bf16", False, 333, 40, 6003, 128, False), ("gated_q8", "bf16", False, 641, 40, 6003, 256, False),
    ("matmul_gx", "bf16", False, 33, 40, 129, 32, False), ("matmul_gx", "bf16", False, 33, 40, 1003, 32, True),
    ("matmul_gx", "bf16", False, 8197, 136, 129, 64, False), ("matmul_gx", "bf16", False, 4101, 40, 4100, 64, True),
    ("matmul_gx", "bf16", False, 4101, 1000, 129, 128, False), ("matmul_gx", "bf16", False, 8197, 40, 4100, 128, True),
    ("matmul_gx", "bf16", False, 8197, 1000, 129, 256, False), ("matmul_gx", "bf16", True, 33, 40, 129, 32, False),
    ("matmul_gx", "bf16", True, 33, 40, 1003, 32, True), ("matmul_gx", "bf16", True, 8197, 136, 129, 64, False),
    ("matmul_gx", "bf16", True, 4101, 40, 4100, 64, True), ("matmul_gx", "bf16", True, 4101, 1000, 129, 128, False),
    ("matmul_gx", "bf16", True, 8197, 40, 4100, 128, True), ("matmul_gx", "bf16", True, 8197, 1000, 129, 256, False),
    ("matmul_gx", "f32", False, 33, 40, 129, 64, False), ("matmul_gx", "f32", False, 33, 40, 520, 64, True),
    ("matmul_gx", "f32", False, 8197, 136, 129, 128, False), ("matmul_gx", "f32", False, 6007, 40, 2049, 128, True),
    ("matmul_gx", "f32", True, 33, 40, 129, 64, False), ("matmul_gx", "f32", True, 33, 40, 520, 64, True),
    ("matmul_gw", "bf16", False, 33, 40, 129, 64, False), ("matmul_gw", "bf16", False, 1025, 40, 129, 64, True),
    ("matmul_gw", "bf16", False, 33, 1000, 4100, 128, False), ("matmul_gw", "bf16", False, 4101, 4104, 129, 128, True),
    ("matmul_gw", "bf16", False, 33, 1000, 8200, 256, False), ("matmul_gw", "bf16", True, 33, 40, 129, 64, False),
    ("matmul_gw", "bf16", True, 1025, 40, 129, 64, True), ("matmul_gw", "bf16", True, 33, 1000, 4100, 128, False),
    ("matmul_gw", "bf16", True, 8197, 40, 4100, 128, True), ("matmul_gw", "bf16", True, 33, 1000, 8200, 256, False),
    ("matmul_gw", "f32", False, 33, 40, 129, 64, False), ("matmul_gw", "f32", False, 333, 40, 129, 64, True),
    ("matmul_gw", "f32", True, 33, 40, 129, 64, False), ("matmul_gw", "f32", True, 333, 40, 129, 64, True),
    ("gated_gx", "bf16", False, 33, 40, 129, 32, False), ("gated_gx", "bf16", False, 33, 40, 520, 32, True),
    ("gated_gx", "bf16", False, 8197, 40, 264, 64, False), ("gated_gx", "bf16", False, 4101, 40, 2049, 64, True),
    ("gated_gx", "bf16", False, 4101, 1000, 129, 128, False), ("gated_gx", "bf16", False, 4101, 40, 4100, 128, True),
    ("gated_gx", "bf16", False, 8197, 1000, 129, 256, False), ("gated_gx", "bf16", False, 8197, 136, 6003, 256, True),
    ("gated_gx", "f32", False, 257, 264, 129, 64, False), ("gated_gx", "f32", False, 33, 40, 129, 64, True),
    ("gated_gx", "f32", False, 8197, 136, 129, 128, False), ("gated_gx", "f32", False, 8197, 40, 520, 128, True),
    ("gated_gw", "bf16", False, 33, 40, 129, 64, False), ("gated_gw", "bf16", False, 1025, 40, 129, 64, True),
    ("gated_gw", "bf16", False, 33, 1000, 2049, 128, False), ("gated_gw", "bf16", False, 4101, 2050, 129, 128, True),
    ("gated_gw", "bf16", False, 33, 1000, 4100, 256, False), ("gated_gw", "bf16", False, 8197, 136, 6003, 256, True),
    ("gated_gw", "f32", False, 33, 40, 129, 64, False), ("gated_gw", "f32", False, 333, 40, 129, 64, True),
    ("matmul_q8", "bf16", False, 333, 8192, 2048, 64, True), ("matmul", "bf16", False, 4101, 6003, 1000, 256, True),
    ("matmul", "bf16", True, 4101, 6003, 1000, 256, True),
    ("matmul_gx", "bf16", False, 4101, 1000, 6003, 256, True), ("matmul_gx", "bf16", True, 4101, 1000, 6003, 256, True),
    ("gated_q8", "bf16", False, 257, 8200, 1003, 64, True),
]


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, shape, scale, dtype):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def _within(got, want, bound, what):
    bad = ~((got.double() - want).abs() <= bound)
    assert got.shape == want.shape and not bool(bad.any()), (what, int(bad.sum()), torch.nonzero(bad)[:3].tolist())


def _sums(pairs):
    """Sum of products of pairs, and of their sizes."""
    return sum(a.double() @ b.double() for a, b in pairs), sum(a.double().abs() @ b.double().abs() for a, b in pairs)


def _forward(product, dtype, odt, transposed, M, K, N, g):
    f32, st = dtype == torch.float32, F.store(odt)
    b, r = _randn(g, (N,), 1.0, odt), _randn(g, (M, N), 1.0, odt)
    if product.endswith("q8"):
        (x, xs), (w, ws), (w2, ws2) = ((torch.randint(-127, 128, (n, K), generator=g, device="cuda", dtype=torch.int8),
                                        torch.rand(n, generator=g, device="cuda") * 0.02 + 1e-3) for n in (M, N, N))
        zd, ud = ((x.double() @ v.double().t()) * xs.double()[:, None] * s.double() for v, s in ((w, ws), (w2, ws2)))
        zb, ub = zd.abs() * 4 * F.U, ud.abs() * 4 * F.U
    else:
        x = _randn(g, (M, K), 1.0, dtype)
        w, w2 = (_randn(g, (N, K) if transposed else (K, N), K ** -0.5, dtype) for _ in range(2))
        zd, zb = _sums([(x, w.t() if transposed else w)])
        zb = zb * F.sum_bound(K, f32)
        if product == "gated":
            ud, ub = _sums([(x, w2)])
            ub = ub * F.sum_bound(K, f32)
    if product.startswith("gated"):
        h = ax.ax_gated_q8(x, xs, w, ws, w2, ws2, out_dtype=odt) if product.endswith("q8") else None
        if h is None:
            h, gp, up = ax.ax_gated(x, w, w2, out_dtype=odt, save=True)
            _within(gp, zd, zb + zd.abs() * st, "g")
            _within(up, ud, ub + ud.abs() * st, "u")
        ad = F.act(zd, "silu")
        _within(h, ad * ud, F.ACT_LIP * zb * (ud.abs() + ub) + ad.abs() * ub + (ad * ud).abs() * (F.ACT_REL + 2 * F.U + st) +
                F.U * zd.abs() * ud.abs(), "h")
        return
    zd, zb = zd + b.double(), zb + 2 * F.U * (zd.abs() + b.double().abs())
    if product == "matmul_q8":
        y = ax.ax_matmul_q8(x, xs, w, ws, bias=b, residual=r, act="relu", out_dtype=odt)
    else:
        y, z = ax.ax_matmul(x, w, bias=b, residual=r, act="relu", transposed=transposed, out_dtype=odt, save=True)
        _within(z, zd, zb + zd.abs() * st, "z")
    yd = torch.relu(zd) + r.double()
    _within(y, yd, zb + 2 * F.U * (yd.abs() + r.double().abs()) + yd.abs() * st, "y")


def _gradient(product, dtype, transposed, M, K, N, g):
    f32, st = dtype == torch.float32, F.store(dtype)
    x, gy = _randn(g, (M, K), 1.0, dtype), _randn(g, (M, N), 1.0, dtype)
    w, w2 = (_randn(g, (N, K) if transposed else (K, N), K ** -0.5, dtype) for _ in range(2))
    if product == "matmul_gx":
        gx = ax.ax_matmul_backward(gy, x, w, transposed=transposed, gw_out=False, gb_out=False)[0]
        want, size = _sums([(gy, w if transposed else w.t())])
        _within(gx, want, size * F.sum_bound(N, f32) + want.abs() * st, "gx")
    elif product == "matmul_gw":
        gw = ax.ax_matmul_backward(gy, x, w, transposed=transposed, gx_out=False, gb_out=False)[1]
        want, size = _sums([(gy.t(), x) if transposed else (x.t(), gy)])
        _within(gw, want, size * F.sum_bound(M, f32) + want.abs() * st, "gw")
    else:  # relu: the slopes are exact, and so are gy u and gy g but for one rounding to the operands' type
        gp, u = _randn(g, (M, N), 1.0, dtype), _randn(g, (M, N), 1.0, dtype)
        grads = gy.double() * u.double() * (gp > 0), gy.double() * torch.relu(gp).double()
        one = 2.0 ** -8 if dtype == torch.bfloat16 else 2 * F.U
        if product == "gated_gx":
            gx = ax.ax_gated_backward(gy, x, w, w2, gp, u, act="relu", gwg_out=False, gwu_out=False)[0]
            want, size = _sums([(grads[0], w.t()), (grads[1], w2.t())])
            _within(gx, want, size * (F.sum_bound(2 * N, f32) + one) + want.abs() * st, "gx")
        else:
            out = ax.ax_gated_backward(gy, x, w, w2, gp, u, act="relu", gx_out=False)[1:]
            for o, v, name in zip(out, grads, ("gwg", "gwu")):
                want, size = _sums([(x.t(), v)])
                _within(o, want, size * (F.sum_bound(M, f32) + one) + want.abs() * st, name)


@pytest.mark.parametrize("product,dt,transposed,M,K,N,rows,sliced", CASES)
def test_tiles(product, dt, transposed, M, K, N, rows, sliced):
    dtype, forward = F.DT[dt], not product.endswith(("gx", "gw"))
    for odt in (torch.bfloat16, torch.float32) if forward else (dtype,):
        plan = ax.ax_probe_product_plan(product, M, K, N, dtype, odt, transposed)
        assert plan["kernel"] == "tiles" and plan["tile"][0] == rows and (plan["slices"] > 1) == sliced, plan
        if forward:
            _forward(product, dtype, odt, transposed, M, K, N, _gen(M + K + N))
    if not forward:
        _gradient(product, dtype, transposed, M, K, N, _gen(M + K + N))

