"""Every tile of the products grouped by expert, with rows in order, looked up through an index and copied first, in every layout, and
every kernel of the products with 4-bit weights.

Sizes are odd and as small as the choice of kernel allows; the test asks for that choice, so that a size whose kernel changes is
noticed and replaced.  References are 64-bit products."""

import pytest
import torch

import ff_common as F
from paper_2002_09481_amd import binding as ax

pytestmark = pytest.mark.gpu

# (product, type, transposed, rows looked up by the tiles, rows, experts, K, N, rows of the tile, workgroups a compute unit)
CASES = [
    ("matmul", "bf16", False, False, 131, 2, 1000, 129, 32, 2), ("matmul", "bf16", False, False, 16411, 3, 72, 41, 64, 2),
    ("matmul", "bf16", False, False, 333, 16, 264, 4100, 64, 3), ("matmul", "bf16", False, False, 8197, 64, 136, 523, 128, 2),
    ("matmul", "bf16", False, False, 8197, 2, 136, 1003, 96, 2),
    ("matmul", "bf16", False, True, 131, 2, 1000, 129, 32, 2), ("matmul", "bf16", False, True, 16411, 3, 72, 41, 64, 2),
    ("matmul", "bf16", False, True, 333, 16, 264, 4100, 64, 3), ("matmul", "bf16", False, True, 8197, 64, 136, 523, 128, 2),
    ("matmul", "bf16", False, True, 8197, 2, 136, 1003, 96, 2),
    ("matmul", "bf16", True, False, 131, 2, 1000, 129, 32, 2), ("matmul", "bf16", True, False, 16411, 3, 72, 41, 64, 2),
    ("matmul", "bf16", True, False, 333, 16, 264, 4100, 64, 3), ("matmul", "bf16", True, False, 8197, 64, 136, 523, 128, 2),
    ("matmul", "bf16", True, False, 8197, 2, 136, 1003, 96, 2),
    ("matmul", "bf16", True, True, 131, 2, 1000, 129, 32, 2), ("matmul", "bf16", True, True, 16411, 3, 72, 41, 64, 2),
    ("matmul", "bf16", True, True, 333, 16, 264, 4100, 64, 3), ("matmul", "bf16", True, True, 8197, 64, 136, 523, 128, 2),
    ("matmul", "bf16", True, True, 8197, 2, 136, 1003, 96, 2),
    ("matmul", "f32", False, False, 131, 2, 520, 129, 64, 2), ("matmul", "f32", True, False, 131, 2, 520, 129, 64, 2),
    ("matmul", "f32", True, False, 16411, 2, 265, 43, 128, 1),
    ("gated", "bf16", False, False, 131, 2, 1000, 129, 32, 2), ("gated", "bf16", False, False, 16411, 3, 72, 41, 64, 2),
    ("gated", "bf16", False, False, 67, 33, 264, 1000, 64, 3), ("gated", "bf16", False, False, 16411, 2, 72, 129, 128, 2),
    ("gated", "bf16", False, False, 1531, 2, 136, 4100, 256, 1),
    ("gated", "bf16", False, True, 131, 2, 1000, 129, 32, 2), ("gated", "bf16", False, True, 16411, 3, 72, 41, 64, 2),
    ("gated", "bf16", False, True, 67, 33, 264, 1000, 64, 3), ("gated", "bf16", False, True, 16411, 2, 72, 129, 128, 2),
    ("gated", "bf16", False, True, 1531, 2, 136, 4100, 256, 1), ("gated", "f32", False, False, 131, 2, 520, 129, 64, 2),
    ("matmul_gx", "bf16", False, False, 131, 2, 129, 1003, 32, 2), ("matmul_gx", "bf16", False, False, 16411, 3, 41, 72, 64, 2),
    ("matmul_gx", "bf16", False, False, 67, 33, 2049, 264, 64, 3), ("matmul_gx", "bf16", False, False, 8197, 64, 523, 137, 128, 2),
    ("matmul_gx", "bf16", False, False, 8197, 2, 1003, 136, 96, 2),
    ("matmul_gx", "bf16", True, False, 131, 2, 129, 1003, 32, 2), ("matmul_gx", "bf16", True, False, 16411, 3, 41, 72, 64, 2),
    ("matmul_gx", "bf16", True, False, 67, 33, 2049, 264, 64, 3), ("matmul_gx", "bf16", True, False, 8197, 64, 523, 137, 128, 2),
    ("matmul_gx", "bf16", True, False, 8197, 2, 1003, 136, 96, 2),
    ("matmul_gx", "f32", False, False, 131, 2, 129, 520, 64, 2), ("matmul_gx", "f32", False, False, 16411, 2, 43, 265, 128, 1),
    ("matmul_gx", "f32", True, False, 131, 2, 129, 520, 64, 2),
    ("gated_gx", "bf16", False, False, 131, 2, 129, 1003, 32, 2), ("gated_gx", "bf16", False, False, 16411, 3, 41, 72, 64, 2),
    ("gated_gx", "bf16", False, False, 67, 33, 2049, 41, 64, 3), ("gated_gx", "bf16", False, False, 8197, 64, 523, 137, 128, 2),
    ("gated_gx", "bf16", False, False, 8197, 2, 1003, 136, 96, 2),
    ("gated_gx", "f32", False, False, 131, 2, 129, 520, 64, 2), ("gated_gx", "f32", False, False, 16411, 2, 43, 265, 128, 1),
    ("matmul_gw", "bf16", False, False, 133, 2, 43, 41, 64, 2), ("matmul_gw", "bf16", False, False, 131, 64, 523, 41, 128, 2),
    ("matmul_gw", "bf16", False, False, 133, 33, 41, 2049, 128, 3), ("matmul_gw", "bf16", False, False, 700, 64, 1003, 129, 256, 1),
    ("matmul_gw", "bf16", True, False, 133, 2, 43, 41, 64, 2), ("matmul_gw", "bf16", True, False, 131, 64, 41, 523, 128, 2),
    ("matmul_gw", "bf16", True, False, 133, 33, 41, 2049, 128, 3), ("matmul_gw", "bf16", True, False, 700, 64, 1003, 129, 256, 1),
    ("matmul_gw", "f32", False, False, 333, 3, 131, 131, 64, 2), ("matmul_gw", "f32", True, False, 333, 3, 131, 131, 64, 2),
    ("gated_gw", "bf16", False, False, 133, 2, 43, 41, 64, 2), ("gated_gw", "bf16", False, False, 131, 33, 523, 41, 128, 2),
    ("gated_gw", "bf16", False, False, 133, 64, 41, 523, 128, 3), ("gated_gw", "bf16", False, False, 333, 8, 1003, 1003, 256, 1),
    ("gated_gw", "f32", False, False, 333, 3, 131, 131, 64, 2),
    ("matmul", "bf16", False, False, 16411, 2, 136, 521, 256, 1), ("matmul", "bf16", False, True, 16411, 2, 136, 521, 256, 1),
    ("matmul_gx", "bf16", False, False, 16411, 2, 521, 136, 256, 1), ("matmul", "bf16", True, False, 16411, 2, 136, 521, 256, 1),
    ("matmul", "bf16", True, True, 16411, 2, 136, 521, 256, 1), ("matmul_gx", "bf16", True, False, 16411, 2, 521, 136, 256, 1),
    ("gated_gx", "bf16", False, False, 16411, 2, 521, 72, 256, 1), ("gated", "bf16", False, False, 1027, 2, 136, 4100, 96, 2),
    ("gated", "bf16", False, True, 1027, 2, 136, 4100, 96, 2),
]
# (gated, type, rows, experts, K, N, kernel, its rows, its columns, its waves)
Q4_CASES = [
    (False, "bf16", 3, 1, 4107, 41, "few", 16, 16, 16), (False, "bf16", 5, 2, 300, 41, "few", 16, 16, 8),
    (False, "bf16", 3, 1, 4107, 8203, "few", 16, 32, 8), (False, "bf16", 17, 1, 4107, 41, "few", 32, 16, 16),
    (False, "bf16", 33, 2, 300, 41, "few", 32, 16, 8), (False, "bf16", 131, 8, 300, 1003, "few", 32, 32, 8),
    (False, "bf16", 67, 2, 300, 41, "few", 64, 16, 8), (False, "bf16", 4099, 64, 300, 41, "few", 64, 32, 8),
    (False, "bf16", 257, 2, 300, 2049, "few", 64, 64, 4), (False, "bf16", 131, 2, 300, 4099, "tiles", 32, 256, 0),
    (False, "bf16", 4099, 8, 300, 265, "tiles", 64, 256, 0), (False, "bf16", 1531, 1, 300, 4099, "written", 128, 128, 0),
    (False, "bf16", 1531, 1, 300, 8203, "written", 256, 256, 0), (False, "bf16", 1301, 2, 300, 1003, "written", 32, 128, 0),
    (False, "bf16", 2051, 1, 300, 1003, "written", 96, 128, 0), (False, "bf16", 8197, 1, 300, 265, "written", 64, 128, 0),
    (False, "f32", 3, 1, 4107, 41, "few", 16, 16, 16), (False, "f32", 5, 2, 300, 41, "few", 16, 16, 8),
    (False, "f32", 3, 1, 300, 8203, "few", 16, 32, 8), (False, "f32", 33, 33, 300, 1003, "few", 16, 64, 8),
    (False, "f32", 33, 2, 300, 41, "few", 32, 16, 8), (False, "f32", 2051, 64, 300, 41, "few", 32, 32, 8),
    (False, "f32", 131, 2, 300, 4099, "tiles", 32, 256, 0), (False, "f32", 4099, 1, 300, 265, "tiles", 64, 256, 0),
    (True, "bf16", 3, 1, 4107, 41, "few", 16, 16, 16), (True, "bf16", 5, 2, 300, 41, "few", 16, 16, 8),
    (True, "bf16", 3, 1, 4107, 8203, "few", 16, 32, 8), (True, "bf16", 17, 1, 4107, 41, "few", 32, 16, 16),
    (True, "bf16", 33, 2, 300, 41, "few", 32, 16, 8), (True, "bf16", 131, 8, 300, 1003, "few", 32, 32, 8),
    (True, "bf16", 67, 2, 300, 41, "few", 64, 16, 8), (True, "bf16", 4099, 64, 300, 41, "few", 64, 32, 8),
    (True, "bf16", 131, 2, 300, 2049, "tiles", 32, 128, 0), (True, "bf16", 4099, 8, 300, 131, "tiles", 64, 128, 0),
    (True, "bf16", 1531, 1, 300, 2049, "written", 128, 128, 0), (True, "bf16", 1531, 1, 300, 4099, "written", 256, 256, 0),
    (True, "bf16", 1301, 2, 300, 523, "written", 32, 128, 0), (True, "bf16", 1301, 2, 300, 1003, "written", 96, 128, 0),
    (True, "bf16", 8197, 1, 300, 131, "written", 64, 128, 0),
    (True, "f32", 3, 1, 4107, 41, "few", 16, 16, 16), (True, "f32", 5, 2, 300, 41, "few", 16, 16, 8),
    (True, "f32", 3, 1, 300, 8203, "few", 16, 32, 8), (True, "f32", 33, 2, 300, 41, "few", 32, 16, 8),
    (True, "f32", 2051, 64, 300, 41, "few", 32, 32, 8), (True, "f32", 131, 2, 300, 2049, "tiles", 32, 128, 0),
    (True, "f32", 4099, 1, 300, 131, "tiles", 64, 128, 0),
]


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, shape, scale, dtype):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def _offsets(rows, E, seed):
    """Ragged experts, the first rows and the last belonging to nobody, an empty expert where there are three or more."""
    g = torch.Generator()
    g.manual_seed(seed)
    cut = torch.sort(torch.randint(2, rows - 1, (E + 1,), generator=g))[0]
    cut[0], cut[-1] = 2, rows - 2
    if E > 2:
        cut[E // 2] = cut[E // 2 + 1]
    return cut.to(torch.int32)


def _per_expert(off, f):
    """f of every expert and its rows, for rows of all: the results one behind the other."""
    cut = off.tolist()
    return [f(e, slice(cut[e], cut[e + 1])) for e in range(len(cut) - 1)]


def _grouped(x, ws, off):
    """Rows of each expert times its matrix, in 64 bits, and the sum of the sizes of the terms; the experts' rows alone."""
    both = _per_expert(off, lambda e, r: (x[r].double() @ ws[e].double(), x[r].double().abs() @ ws[e].double().abs()))
    return torch.cat([b[0] for b in both]), torch.cat([b[1] for b in both])


def _within(got, want, bound, what):
    bad = ~((got.double() - want).abs() <= bound)
    assert got.shape == want.shape and not bool(bad.any()), (what, int(bad.sum()), torch.nonzero(bad)[:3].tolist())


@pytest.mark.parametrize("product,dt,transposed,found,rows,E,K,N,high,per_cu", CASES)
def test_tiles(product, dt, transposed, found, rows, E, K, N, high, per_cu):
    dtype, f32, g = F.DT[dt], dt == "f32", _gen(rows + K + N)
    X = rows // 2 + 1
    plan = ax.ax_probe_experts_plan(product, rows, E, K, N, dtype, transposed, x_rows=X if found else None)
    assert (plan["kernel"], plan["tile"][0], plan["per_cu"], plan["found"]) == ("tiles", high, per_cu, found), plan
    off = _offsets(rows, E, rows + E)
    mine, st = slice(int(off[0]), int(off[-1])), F.store(dtype)
    x = _randn(g, (X if found else rows, K), 1.0, dtype)
    index = torch.randint(0, X, (rows,), generator=g, device="cuda", dtype=torch.int32) if found else None
    xr = x[index.long()] if found else x
    w, w2 = (_randn(g, (E, N, K) if transposed else (E, K, N), K ** -0.5, dtype) for _ in range(2))
    mat = lambda v: v.transpose(1, 2) if transposed else v  # noqa: E731
    offsets = off.cuda()
    left = lambda t: bool((t[:mine.start] == 7).all()) and bool((t[mine.stop:] == 7).all())  # noqa: E731
    mark = lambda n: torch.full((rows, n), 7.0, dtype=dtype, device="cuda")  # noqa: E731
    if product == "matmul":
        y, z = ax.ax_matmul_experts(x, w, offsets, index, act="relu", transposed=transposed, y_out=mark(N), z_out=mark(N))
        zd, size = _grouped(xr, mat(w), off)
        zb = size * F.sum_bound(K, f32) + zd.abs() * st
        _within(z[mine], zd, zb, "z")
        _within(y[mine], torch.relu(zd), zb, "y")
        assert left(y) and left(z)
    elif product == "gated":
        h, gp, up = ax.ax_gated_experts(x, w, w2, offsets, index, act="relu", h_out=mark(N), g_out=mark(N), u_out=mark(N))
        (gd, gs), (ud, us), s = _grouped(xr, w, off), _grouped(xr, w2, off), F.sum_bound(K, f32)
        _within(gp[mine], gd, gs * s + gd.abs() * st, "g")
        _within(up[mine], ud, us * s + ud.abs() * st, "u")
        hd = torch.relu(gd) * ud
        _within(h[mine], hd, gs * s * (ud.abs() + us * s) + gd.abs() * us * s + hd.abs() * (2 * F.U + st), "h")
        assert left(h) and left(gp) and left(up)
    else:
        gy = _randn(g, (rows, N), 1.0, dtype)
        if product.startswith("matmul"):
            grads, one, names = [gy], 0.0, ("gw",)
            out = ax.ax_matmul_experts_backward(gy, x, w, offsets, transposed=transposed, gx_out=mark(K))
        else:  # relu: slopes are exact, gy u and gy g are but for one rounding to the operands' type
            gp, u = _randn(g, (rows, N), 1.0, dtype), _randn(g, (rows, N), 1.0, dtype)
            grads, names = [gy.double() * u.double() * (gp > 0), gy.double() * torch.relu(gp).double()], ("gwg", "gwu")
            one = 2 * F.U if f32 else 2.0 ** -8
            out = ax.ax_gated_experts_backward(gy, x, w, w2, gp, u, offsets, act="relu", gx_out=mark(K))
        if product.endswith("gx"):
            parts = [_grouped(v, mat(m).transpose(1, 2), off) for v, m in zip(grads, (w, w2))]
            want, size = sum(p[0] for p in parts), sum(p[1] for p in parts)
            _within(out[0][mine], want, size * (F.sum_bound(len(grads) * N, f32) + one) + want.abs() * st, "gx")
            assert left(out[0])
        else:
            for o, v, name in zip(out[1:], grads, names):
                o = mat(o)
                for e, (got, want, size, n) in enumerate(_per_expert(off, lambda e, r: (
                        o[e], x[r].double().t() @ v[r].double(), x[r].double().abs().t() @ v[r].double().abs(), r.stop - r.start))):
                    _within(got, want, size * (F.sum_bound(max(n, 1), f32) + one) + want.abs() * st, (name, e))


@pytest.mark.parametrize("indexed", [False, True])
@pytest.mark.parametrize("gated,dt,rows,E,K,N,kernel,high,cols,waves", Q4_CASES)
def test_q4_kernels(gated, dt, rows, E, K, N, kernel, high, cols, waves, indexed):
    dtype, f32, g, X = F.DT[dt], dt == "f32", _gen(rows + K + N), rows // 2 + 1
    plan = ax.ax_probe_q4_plan(gated, rows, E, K, N, 64, dtype, x_rows=X if indexed else None)
    assert (plan["kernel"], plan["tile"], plan["waves"]) == (kernel, (high, cols), waves), plan
    off = _offsets(rows, E, rows + E) if E > 1 else torch.tensor([0, rows])
    mine, st = slice(int(off[0]), int(off[-1])), F.store(dtype)
    x = _randn(g, (X if indexed else rows, K), 1.0, dtype)
    index = torch.randint(0, X, (rows,), generator=g, device="cuda", dtype=torch.int32) if indexed else None
    xr = x[index.long()] if indexed else x
    shape, scale_shape = ((E, N, K), (E, N, -(-K // 64))) if E > 1 else ((N, K), (N, -(-K // 64)))
    ws, values, most = [], [], []
    for _ in range(1 + gated):
        codes = torch.randint(-8, 8, shape, generator=g, device="cuda", dtype=torch.int8)
        scales = ((torch.rand(scale_shape, generator=g, device="cuda") + 0.1) * K ** -0.5 / 4).to(torch.bfloat16)
        wide = scales.double().repeat_interleave(64, dim=-1)[..., :K]
        ws.append(ax.ax_pack_q4(codes, scales, group=64))
        values.append((codes.double() * wide).view(E, N, K).transpose(1, 2))
        most.append((wide * 55).view(E, N, K).transpose(1, 2))
    kw = dict(offsets=off.to(torch.int32).cuda() if E > 1 else None, tokens=index)
    y = torch.full((rows, N), 7.0, dtype=dtype, device="cuda")

    def sums(i):
        """Sums and their bounds.  Tiles of bf16 add 24 to the codes (31 then at most) and take 24 off; written weights are rounded once."""
        z, size = _grouped(xr, values[i], off)
        if kernel == "tiles" and not f32:
            return z, _grouped(xr, most[i], off)[1] * F.sum_bound(K)
        return z, size * (F.sum_bound(K, f32) + (2.0 ** -8 * 1.01 if kernel == "written" else 0))

    zd, zb = sums(0)
    if not gated:
        ax.ax_matmul_q4(x, ws[0], y_out=y, **kw)
        _within(y[mine], zd, zb + zd.abs() * (2 * F.U + st), "y")
    else:
        ax.ax_gated_q4(x, ws[0], ws[1], act="relu", h_out=y, **kw)
        ud, ub = sums(1)
        hd = torch.relu(zd) * ud
        _within(y[mine], hd, zb * (ud.abs() + ub) + zd.abs() * ub + hd.abs() * (2 * F.U + st), "h")
    assert bool((y[:mine.start] == 7).all()) and bool((y[mine.stop:] == 7).all())
