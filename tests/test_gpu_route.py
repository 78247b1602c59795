"""The router and the sum of the experts' rows against 64-bit forms: ties, masks, rows that are masked altogether, infinities and
NaN, the order of rows, gradients, odd sizes and pitches."""

import math

import pytest
import torch

import ff_common as F
from paper_2002_09481_amd import binding as ax

pytestmark = pytest.mark.gpu

INF = float("inf")


def plain_choice(logits, k, normalize):
    """Experts, weights (float64) of each token, one by one."""
    x = logits.double()
    T, E = x.shape
    experts, weights = torch.full((T, k), -1, dtype=torch.int32), torch.zeros((T, k), dtype=torch.float64)
    for t in range(T):
        row = x[t].tolist()
        alive = [e for e in range(E) if row[e] > -INF]  # (a NaN compares false)
        chosen = sorted(alive, key=lambda e: (-row[e], e))[:k]
        if not chosen:
            continue
        m = row[chosen[0]]
        ex = lambda e: 1.0 if row[e] == m else math.exp(row[e] - m)  # noqa: E731
        total = sum(ex(e) for e in (chosen if normalize else alive))
        if any(v != v for v in row):
            total = float("nan")
        for j, e in enumerate(chosen):
            experts[t, j], weights[t, j] = e, ex(e) / total
    return experts, weights


def plain_order(experts, E):
    """Offsets, rows, tokens of the choices by (expert, token, choice)."""
    T, k = experts.shape
    items = sorted((int(experts[t, j]), t, j) for t in range(T) for j in range(k) if experts[t, j] >= 0)
    rows, tokens, counts = torch.full((T, k), -1, dtype=torch.int32), torch.full((T * k,), -1, dtype=torch.int32), [0] * E
    for r, (e, t, j) in enumerate(items):
        rows[t, j], tokens[r] = r, t
        counts[e] += 1
    offsets = torch.tensor([sum(counts[:e]) for e in range(E + 1)], dtype=torch.int32)
    return offsets, rows, tokens


def check_route(logits, k, normalize, out=None):
    experts, weights, offsets, rows, tokens = out or ax.ax_route(logits.cuda(), k, normalize=normalize)
    we, ww = plain_choice(logits, k, normalize)
    assert torch.equal(experts.cpu(), we)
    # differences of logits within 40 and their exponentials within 40 + 4 roundings, a sum of up to E / 8 steps, a quotient
    bound = ww * (48 + logits.shape[1] / 8 + 8) * 2 * F.U
    nan = torch.isnan(ww)
    assert torch.equal(torch.isnan(weights.cpu()), nan)
    F.assert_within(weights.cpu().double().masked_fill(nan, 0), ww.masked_fill(nan, 0), bound.masked_fill(nan, 0) + 1e-30)
    for got, want in zip((offsets, rows, tokens), plain_order(we, logits.shape[1])):
        assert got.dtype == torch.int32 and torch.equal(got.cpu(), want)
    return experts, weights, offsets, rows, tokens


@pytest.mark.parametrize("normalize", [True, False])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 64, 6), (2, 7, 7), (63, 60, 4), (64, 64, 16), (65, 65, 3), (130, 128, 8), (97, 129, 5),
                                   (70, 256, 2), (16, 257, 9), (17, 1000, 16), (33, 1024, 1), (600, 5, 2), (1500, 33, 8)])
def test_route(T, E, k, dt, normalize):
    g = F.gen(T * 13 + E)
    logits = F.randn(g, (T, E), 2.0, F.DT[dt])  # (bf16: many ties)
    check_route(logits, k, normalize)


@pytest.mark.parametrize("T", [40, 70000])
def test_order_of_many_tokens(T):
    """Several blocks, each of several turns: against a stable sort."""
    g = F.gen(T)
    E, k = 19, 3
    logits = F.randn(g, (T, E), 1.0, torch.bfloat16).cuda()
    experts, _, offsets, rows, tokens = ax.ax_route(logits, k)
    by, order = torch.sort(experts.reshape(-1).cpu().long(), stable=True)
    assert torch.equal(tokens.cpu().long(), order // k)
    assert torch.equal(offsets.cpu().long(), torch.searchsorted(by, torch.arange(E + 1)))
    assert torch.equal(rows.cpu().long().reshape(-1)[order], torch.arange(T * k))


@pytest.mark.parametrize("normalize", [True, False])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_masks_infinities_and_ties(dt, normalize):
    g = F.gen(3)
    x = F.randn(g, (80, 24), 1.0, F.DT[dt])
    low = torch.finfo(F.DT[dt]).min
    x[0] = -INF  # masked altogether
    x[1] = -INF
    x[1, 5] = 1.0  # one left
    x[2, 3:] = -INF  # three left for four choices
    x[3] = 0.0  # all equal
    x[4] = low  # masked with the lowest value: still numbers
    x[5, 7] = INF
    x[6, 2] = x[6, 9] = INF
    x[7, 11] = float("nan")
    x[8] = float("nan")
    x[9, 1:] = low
    x[10, 4], x[10, 5] = 0.0, -0.0
    x[11] = -0.0
    x[11, 3] = 0.0
    x[12, 20] = -INF
    experts, weights, *_ = check_route(x, 4, normalize)
    assert weights[0].tolist() == [0.0] * 4 and experts[0].tolist() == [-1] * 4
    assert experts[3].tolist() == [0, 1, 2, 3] and experts[11].tolist() == [0, 1, 2, 3]
    assert weights[6].tolist() == [0.5, 0.5, 0.0, 0.0]


def test_every_token_masked():
    out = ax.ax_route(torch.full((5, 9), -INF, device="cuda"), 2)
    assert bool((out[0] == -1).all()) and not bool(out[1].any()) and not bool(out[2].any())
    assert bool((out[3] == -1).all()) and bool((out[4] == -1).all())


def test_no_tokens():
    out = ax.ax_route(torch.empty((0, 9), device="cuda"), 2, offsets_out=torch.full((10,), 7, dtype=torch.int32, device="cuda"))
    assert out[0].shape == (0, 2) and out[4].shape == (0,) and out[2].tolist() == [0] * 10
    assert ax.ax_route_backward(out[1], torch.empty((0, 9), device="cuda"), out[0], out[1]).shape == (0, 9)


@pytest.mark.parametrize("offset,pad", [(0, 8), (1, 6), (3, 0)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_pitches_of_logits(dt, offset, pad):
    g, T, E, k = F.gen(5), 150, 50, 3
    wide = F.randn(g, (T, E + offset + pad), 1.0, F.DT[dt]).cuda()
    inner = wide[:, offset:offset + E]
    want = ax.ax_route(inner.contiguous(), k)
    got = ax.ax_route(inner, k)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    gw = F.randn(g, (T, k)).cuda()
    buf = torch.full_like(wide, 5.0)
    for normalize in (True, False):
        ref = ax.ax_route_backward(gw, inner.contiguous(), want[0], want[1], normalize=normalize)
        ax.ax_route_backward(gw, inner, want[0], want[1], normalize=normalize, glogits_out=buf[:, offset:offset + E])
        assert torch.equal(buf[:, offset:offset + E], ref)
        assert bool((buf[:, :offset] == 5).all()) and bool((buf[:, offset + E:] == 5).all())


@pytest.mark.parametrize("normalize", [True, False])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (5, 64, 6), (40, 7, 7), (33, 60, 4), (100, 128, 8), (50, 200, 16), (19, 257, 3), (9, 1024, 16)])
def test_route_gradient(T, E, k, dt, normalize):
    g, dtype = F.gen(T + E), F.DT[dt]
    logits, gw = F.randn(g, (T, E), 1.0, dtype), F.randn(g, (T, k))
    if T > 3:
        logits[1] = -INF
        logits[2, 1:] = -INF
    experts, weights, *_ = ax.ax_route(logits.cuda(), k, normalize=normalize)
    got = ax.ax_route_backward(gw.cuda(), logits.cuda(), experts, weights, normalize=normalize)
    x = logits.double()
    x.requires_grad_()
    e = experts.cpu().long()
    p = torch.softmax(x, dim=1).nan_to_num() if not normalize else None
    top = torch.gather(x, 1, e.clamp(min=0)).masked_fill(e < 0, -INF)
    w = torch.softmax(top, dim=1).nan_to_num() if normalize else torch.gather(p, 1, e.clamp(min=0)).masked_fill(e < 0, 0.0)
    (w * gw.double()).sum().backward()
    want = x.grad.nan_to_num()
    # weights and softmax within 64 + E / 4 roundings, the inner sum of k terms and the product
    size = weights.cpu().double() * gw.double().abs()
    inner = size.sum(dim=1, keepdim=True)
    full = torch.zeros_like(want).scatter_add_(1, e.clamp(min=0), size.masked_fill(e < 0, 0.0))
    q = torch.softmax(x.detach(), dim=1).nan_to_num() if not normalize else torch.zeros_like(want).scatter_add_(
        1, e.clamp(min=0), weights.cpu().double().masked_fill(e < 0, 0.0))
    F.assert_within(got, want, (full + q * inner) * (80 + E / 4 + 2 * k) * 2 * F.U + want.abs() * F.store(dtype) + 1e-30)


def test_route_gradient_against_differences():
    g, T, E, k, e = F.gen(9), 12, 10, 3, 1e-5
    logits, gw, d = F.randn(g, (T, E)), F.randn(g, (T, k)), F.randn(g, (T, E)).double()
    for normalize in (True, False):
        experts, weights, *_ = ax.ax_route(logits.cuda(), k, normalize=normalize)
        got = (ax.ax_route_backward(gw.cuda(), logits.cuda(), experts, weights, normalize=normalize).cpu().double() * d)
        idx = experts.cpu().long()

        def loss(s):
            x = logits.double() + s * d
            w = torch.softmax(torch.gather(x, 1, idx), dim=1) if normalize else torch.gather(torch.softmax(x, dim=1), 1, idx)
            return float((w * gw.double()).sum())

        slope = (loss(e) - loss(-e)) / (2 * e)
        third = abs(loss(1e-2) - 2 * loss(5e-3) + 2 * loss(-5e-3) - loss(-1e-2)) / (2 * 5e-3 ** 3)
        assert abs(float(got.sum()) - slope) <= e * e * third + 1e-15 * T / e + float(got.abs().sum()) * 200 * F.U


def test_route_gradient_of_very_many_tokens():
    """More than a launch can count the threads of."""
    T, kw = (1 << 28) + 5, dict(device="cuda")
    logits, experts = torch.zeros((T, 1), dtype=torch.bfloat16, **kw), torch.zeros((T, 1), dtype=torch.int32, **kw)
    weights, gw = torch.full((T, 1), 0.5, **kw), torch.full((T, 1), 2.0, **kw)
    out = ax.ax_route_backward(gw, logits, experts, weights, glogits_out=torch.full_like(logits, 7.0))
    assert int((out == 0.5).sum()) == T  # 0.5 (2 - 1)


def test_route_gradient_of_nan_shows():
    x = torch.zeros((3, 20))
    x[1, 4] = float("nan")
    for normalize in (True, False):
        experts, weights, *_ = ax.ax_route(x.cuda(), 2, normalize=normalize)
        gl = ax.ax_route_backward(torch.ones((3, 2), device="cuda"), x.cuda(), experts, weights, normalize=normalize)
        assert bool(torch.isnan(gl[1]).any()) and bool(torch.isfinite(gl[[0, 2]]).all())


# ---- the sum of the experts' rows --------------------------------------------------------------


def _plain_combine(h, rows, weights, r):
    T, k = rows.shape
    ok = (rows >= 0) & (rows < h.shape[0])
    hv = h.double()[rows.long().clamp(0, max(h.shape[0] - 1, 0))] * ok[:, :, None] if h.shape[0] else torch.zeros((T, k, h.shape[1])).double()
    hv = torch.where(ok[:, :, None], hv, torch.zeros_like(hv))
    w = (torch.ones((T, k)) if weights is None else weights).double() * ok
    t = w[:, :, None] * hv
    y = t.sum(dim=1) + (0 if r is None else r.double())
    size = t.abs().sum(dim=1) + (0 if r is None else r.double().abs())
    return y, size


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T,k,cols", [(1, 1, 1), (1, 6, 2048), (5, 4, 7), (37, 2, 64), (64, 3, 1000), (130, 8, 129), (9, 16, 4096), (3, 5, 8200)])
def test_combine(T, k, cols, dt):
    g, dtype = F.gen(T + k + cols), F.DT[dt]
    h, r = F.randn(g, (T * k, cols), 1.0, dtype), F.randn(g, (T, cols), 1.0, dtype)
    rows = torch.randperm(T * k, generator=g).to(torch.int32).view(T, k)
    w, gy = torch.rand((T, k), generator=g), F.randn(g, (T, cols), 1.0, dtype)
    if T > 4:  # dropped choices, and rows outside
        rows[0], rows[1, 0], rows[2, k - 1], rows[3, 0] = -1, -1, T * k, 2 ** 31 - 1
    for weights, res in ((w, r), (None, None), (w, None)):
        y, size = _plain_combine(h, rows, weights, res)
        dev = [None if t is None else t.cuda() for t in (weights, res)]
        got = ax.ax_combine(h.cuda(), rows.cuda(), *dev)
        F.assert_within(got, y, size * (k + 2) * F.U + y.abs() * F.store(dtype))
    out = ax.ax_combine(h.cuda(), rows.cuda(), w.cuda(), residual=r.cuda())
    rc = r.cuda()
    assert ax.ax_combine(h.cuda(), rows.cuda(), w.cuda(), residual=rc, y_out=rc) is rc and torch.equal(rc, out)

    for weights in (w, None):
        wc = None if weights is None else weights.cuda()
        gh, gw = ax.ax_combine_backward(gy.cuda(), h.cuda(), rows.cuda(), wc, gh_out=torch.full_like(h, 9.0).cuda())
        wh = torch.full_like(h, 9.0).double()
        ok = (rows >= 0) & (rows < T * k)
        ww = torch.ones((T, k)).double() if weights is None else weights.double()
        for t in range(T):
            for j in range(k):
                if ok[t, j]:
                    wh[int(rows[t, j])] = ww[t, j] * gy[t].double()
        F.assert_within(gh, wh, wh.abs() * (F.store(dtype) + 2 * F.U), "gh")
        hv = torch.where(ok[:, :, None], h.double()[rows.long().clamp(0, T * k - 1)], torch.zeros(()).double())
        terms = hv * gy.double()[:, None, :]
        F.assert_within(gw, terms.sum(dim=2), terms.abs().sum(dim=2) * (cols / 64 + 24) * 2 * F.U, "gweights")
        only = ax.ax_combine_backward(gy.cuda(), h.cuda(), rows.cuda(), wc, gh_out=False)
        assert only[0] is None and torch.equal(only[1], gw)
        only = ax.ax_combine_backward(gy.cuda(), h.cuda(), rows.cuda(), wc, gh_out=torch.full_like(h, 9.0).cuda(), gweights_out=False)
        assert only[1] is None and torch.equal(only[0], gh)


@pytest.mark.parametrize("offset,pad", [(0, 8), (1, 6), (8, 3)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_combine_pitches(dt, offset, pad):
    g, T, k, cols = F.gen(6), 21, 3, 200
    wide = lambda n: F.randn(g, (n, cols + offset + pad), 1.0, F.DT[dt]).cuda()  # noqa: E731
    inner = lambda t: t[:, offset:offset + cols]  # noqa: E731
    H, R, Y, GY = wide(T * k), wide(T), wide(T), wide(T)
    rows, w = torch.randperm(T * k, generator=g).to(torch.int32).view(T, k).cuda(), torch.rand((T, k), generator=g).cuda()
    old = Y.clone()
    ax.ax_combine(inner(H), rows, w, residual=inner(R), y_out=inner(Y))
    assert torch.equal(inner(Y), ax.ax_combine(inner(H).contiguous(), rows, w, residual=inner(R).contiguous()))
    inner(Y)[:] = inner(old)
    assert torch.equal(Y, old)
    gh, gw = ax.ax_combine_backward(inner(GY), inner(H), rows, w, gh_out=inner(H.clone()))
    wh, ww = ax.ax_combine_backward(inner(GY).contiguous(), inner(H).contiguous(), rows, w)
    assert torch.equal(gh, wh) and torch.equal(gw, ww)


def test_combine_without_rows_or_tokens():
    h, r = torch.empty((0, 24), device="cuda"), torch.ones((3, 24), device="cuda")
    rows = torch.full((3, 2), -1, dtype=torch.int32, device="cuda")
    assert torch.equal(ax.ax_combine(h, rows, residual=r), r) and not bool(ax.ax_combine(h, rows).any())
    gh, gw = ax.ax_combine_backward(r, h, rows)
    assert gh.shape == (0, 24) and not bool(gw.any())
    none = torch.empty((0, 2), dtype=torch.int32, device="cuda")
    assert ax.ax_combine(r, none).shape == (0, 24)


def test_combine_leaves_out_what_a_dropped_row_holds():
    h = torch.full((4, 40), float("nan"), device="cuda")
    h[1] = 2.0
    rows = torch.tensor([[1, -1], [4, 1]], dtype=torch.int32, device="cuda")
    w = torch.tensor([[0.5, float("nan")], [float("inf"), 3.0]], device="cuda")
    assert ax.ax_combine(h, rows, w).cpu().tolist() == [[1.0] * 40, [6.0] * 40]
