"""What the operators of a block of experts and of 4-bit weights refuse, on the host, before any device work."""

import ctypes
import os

import pytest
import torch

from paper_2002_09481_amd import binding as ax

pytestmark = pytest.mark.skipif(not os.path.exists(ax.LIB_PATH), reason="libaxconv.so not built")
P, ODD, HALF = ctypes.c_void_p(4096), ctypes.c_void_p(4097), ctypes.c_void_p(4098)
R, BIG = ctypes.byref, 1 << 40


def changed(d, kw):
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def route(**kw):
    return changed(ax.ax_route_desc_t(5000, 16, 16, 2, 1, 1), kw)


def experts(**kw):
    return changed(ax.ax_experts_desc_t(400, 100, 64, 32, 32, 64, 64, 32, 4, 1, 0, 0, 1, 0), kw)


def combine(**kw):
    return changed(ax.ax_combine_desc_t(100, 200, 64, 64, 64, 64, 64, 2, 1), kw)


def q4(**kw):
    return changed(ax.ax_q4_desc_t(4000, 100, 64, 32, 32, 64, 64, 4, 32, 1, 0, 1, 0), kw)


def null_each(call, n, skip=()):
    """Every pointer NULL in turn gives -1."""
    for k in range(n):
        if k not in skip:
            assert call(*[None if i == k else P for i in range(n)]) == -1, k


def odd_each(call, n, bad=ODD, skip=()):
    for k in range(n):
        if k not in skip:
            assert call(*[bad if i == k else P for i in range(n)]) == -7, k


@pytest.mark.parametrize("bad,code", [(dict(tokens=-1), -2), (dict(experts=0), -2), (dict(experts=1025, ld=1025), -2), (dict(k=0), -2), (dict(k=17), -2),
                                      (dict(experts=8, k=9), -2), (dict(ld=15), -2), (dict(ld=1 << 21), -2), (dict(tokens=(1 << 29) + 1), -2),
                                      (dict(dtype=2), -8), (dict(normalize=2), -8)])
def test_router_descriptions(bad, code):
    L = ax.lib()
    assert L.ax_route(R(route(**bad)), *[P] * 7, BIG, None) == code and L.ax_route_workspace_bytes(R(route(**bad))) == 0
    assert L.ax_route_backward(R(route(**bad)), *[P] * 5, 16, None) == code


def test_router_pointers():
    L, d = ax.lib(), route()
    need = L.ax_route_workspace_bytes(R(d))
    assert need > 0 and L.ax_route_workspace_bytes(R(route(tokens=3))) == 0
    go = lambda *a: L.ax_route(R(d), *a, P, need, None)  # noqa: E731
    null_each(go, 6)
    odd_each(go, 6)
    odd_each(go, 6, HALF, skip=(0,))  # (bf16 logits may start there)
    assert L.ax_route(None, *[P] * 7, need, None) == -1
    assert L.ax_route(R(d), *[P] * 6, P, need - 1, None) == -5 and L.ax_route(R(d), *[P] * 6, None, need, None) == -5
    assert L.ax_route(R(d), *[P] * 6, ctypes.c_void_p(4096 + 16), need, None) == -5
    back = lambda *a: L.ax_route_backward(R(route(normalize=0)), *a, 16, None)  # noqa: E731
    null_each(back, 5)
    odd_each(back, 5)
    assert L.ax_route_backward(R(d), *[P] * 5, 15, None) == -2 and L.ax_route_backward(None, *[P] * 5, 16, None) == -1
    assert L.ax_route_backward(R(route(tokens=0)), *[None] * 5, 16, None) == 0


@pytest.mark.parametrize("bad,code", [(dict(rows=-1), -2), (dict(rows=(1 << 30) + 1), -2), (dict(x_rows=-1), -2), (dict(N=0), -2), (dict(K=0), -2),
                                      (dict(experts=0), -2), (dict(experts=1025), -2), (dict(N=1 << 29, w_ld=1 << 29), -2), (dict(x_ld=31), -2),
                                      (dict(w_ld=63), -2), (dict(y_ld=63), -2), (dict(indexed=0), -2), (dict(dtype=2), -8), (dict(act=4), -8),
                                      (dict(act=-1), -8), (dict(w_transposed=2), -8), (dict(indexed=2), -8), (dict(unaligned=-1), -8)])
def test_expert_descriptions(bad, code):
    L, d = ax.lib(), experts(**bad)
    assert L.ax_matmul_experts(R(d), *[P] * 7, BIG, None) == code and L.ax_matmul_experts_workspace_bytes(R(d)) == 0
    assert L.ax_gated_experts(R(d), *[P] * 9, BIG, None) == code and L.ax_gated_experts_workspace_bytes(R(d)) == 0
    assert L.ax_matmul_experts_backward(R(d), *[P] * 9, BIG, None) == code and L.ax_matmul_experts_backward_workspace_bytes(R(d)) == 0
    assert L.ax_gated_experts_backward(R(d), *[P] * 12, BIG, None) == code and L.ax_gated_experts_backward_workspace_bytes(R(d)) == 0


def test_expert_pointers():
    L, d = ax.lib(), experts()
    mm = lambda *a: L.ax_matmul_experts(R(d), *a, P, BIG, None)  # noqa: E731
    null_each(mm, 6, skip=(5,))
    odd_each(mm, 6)
    odd_each(mm, 6, HALF, skip=(4, 5))  # (outputs may start at any element)
    assert L.ax_matmul_experts(R(experts(indexed=0, x_rows=400)), HALF, None, P, P, P, P, P, BIG, None) == -7
    assert L.ax_matmul_experts(R(experts(indexed=0, x_rows=400)), P, P, P, P, P, P, P, BIG, None) == -1  # an index that is not said
    copied = experts(unaligned=1)
    need = L.ax_matmul_experts_workspace_bytes(R(copied))
    assert need >= 400 * 64 and L.ax_matmul_experts(R(copied), *[P] * 6, P, need - 1, None) == -5
    assert L.ax_matmul_experts_workspace_bytes(R(d)) == 0  # read in place, rows found through the index
    gated = lambda *a: L.ax_gated_experts(R(d), *a, P, BIG, None)  # noqa: E731
    null_each(gated, 8)  # (one projection without the other)
    odd_each(gated, 8)
    assert L.ax_gated_experts(R(experts(w_transposed=1, w_ld=32)), *[P] * 9, BIG, None) == -8
    back = lambda *a: L.ax_matmul_experts_backward(R(experts(act=2)), *a, P, BIG, None)  # noqa: E731
    null_each(back, 8, skip=(6, 7))
    odd_each(back, 8)
    assert back(P, P, P, P, P, P, None, None) == -1
    assert L.ax_matmul_experts_backward(R(experts(gx_ld=31)), *[P] * 9, BIG, None) == -2
    gback = lambda *a: L.ax_gated_experts_backward(R(d), *a, P, BIG, None)  # noqa: E731
    null_each(gback, 11, skip=(8,))
    odd_each(gback, 11)
    assert gback(*[P] * 8, None, None, None) == -1
    assert L.ax_gated_experts_backward(R(d), *[P] * 11, P, L.ax_gated_experts_backward_workspace_bytes(R(d)) - 1, None) == -5
    none = experts(rows=0)
    assert L.ax_matmul_experts(R(none), *[None] * 7, 0, None) == 0 and L.ax_matmul_experts_workspace_bytes(R(none)) == 0


@pytest.mark.parametrize("bad,code", [(dict(tokens=-1), -2), (dict(h_rows=-1), -2), (dict(cols=0), -2), (dict(k=0), -2), (dict(k=17), -2),
                                      (dict(h_ld=63), -2), (dict(y_ld=63), -2), (dict(tokens=(1 << 29) + 1), -2), (dict(dtype=2), -8)])
def test_sum_descriptions(bad, code):
    L, d = ax.lib(), combine(**bad)
    assert L.ax_combine(R(d), *[P] * 6) == code and L.ax_combine_backward(R(d), *[P] * 7) == code


def test_sum_pointers():
    L, d = ax.lib(), combine()
    go = lambda *a: L.ax_combine(R(d), *a, None)  # noqa: E731
    null_each(go, 5, skip=(2, 3))
    odd_each(go, 5)
    assert L.ax_combine(R(combine(residual_ld=3)), *[P] * 6) == -2 and L.ax_combine(None, *[P] * 6) == -1
    back = lambda *a: L.ax_combine_backward(R(d), *a, None)  # noqa: E731
    null_each(back, 6, skip=(3, 4, 5))
    odd_each(back, 6)
    assert back(P, P, P, P, None, None) == -1
    assert L.ax_combine_backward(R(combine(gh_ld=3)), *[P] * 7) == -2
    assert L.ax_combine(R(combine(tokens=0)), *[None] * 6) == 0


WEIGHTS = [(dict(experts=0), -2), (dict(experts=1025), -2), (dict(N=0), -2), (dict(K=0), -2), (dict(N=1 << 31), -2), (dict(group=16), -8), (dict(group=96), -8),
           (dict(N=1 << 20, K=1 << 20), -2)]


@pytest.mark.parametrize("bad,code", WEIGHTS)
def test_4_bit_weights(bad, code):
    L = ax.lib()
    a = dict(dict(experts=2, N=64, K=32, group=32), **bad)
    size = (a["experts"], a["N"], a["K"])
    assert L.ax_quantize_q4(P, 1, 1 << 20, *size, a["group"], P, P, None) == code
    assert L.ax_pack_q4(P, P, *size, a["group"], P, P, None) == code and L.ax_q4_values(P, P, *size, a["group"], P, None) == code
    assert L.ax_q4_scales_bytes(*size, a["group"]) == 0
    if "group" not in bad:
        assert L.ax_q4_codes_bytes(*size) == 0


def test_4_bit_weight_pointers():
    L, size = ax.lib(), (2, 64, 32, 32)
    assert L.ax_q4_codes_bytes(2, 64, 32) == 2 * 4 * 1024 and L.ax_q4_scales_bytes(2, 64, 32, 32) == 2 * 4 * 4 * 16 * 2
    assert L.ax_quantize_q4(P, 2, 32, *size, P, P, None) == -8 and L.ax_quantize_q4(P, 1, 31, *size, P, P, None) == -2
    null_each(lambda w, c, s: L.ax_quantize_q4(w, 1, 32, *size, c, s, None), 3)
    odd_each(lambda w, c, s: L.ax_quantize_q4(w, 1, 32, *size, c, s, None), 3)
    null_each(lambda c, s, o, p: L.ax_pack_q4(c, s, *size, o, p, None), 4)
    odd_each(lambda c, s, o, p: L.ax_pack_q4(c, s, *size, o, p, None), 4, skip=(0,))
    null_each(lambda c, s, o: L.ax_q4_values(c, s, *size, o, None), 3)
    odd_each(lambda c, s, o: L.ax_q4_values(c, s, *size, o, None), 3)


@pytest.mark.parametrize("bad,code", WEIGHTS[:-1] + [(dict(rows=-1), -2), (dict(x_rows=-1), -2), (dict(indexed=0), -2), (dict(x_ld=31), -2), (dict(y_ld=63), -2),
                                                (dict(dtype=2), -8), (dict(act=4), -8), (dict(indexed=2), -8), (dict(unaligned=2), -8)])
def test_4_bit_product_descriptions(bad, code):
    L, d = ax.lib(), q4(**bad)
    assert L.ax_matmul_q4(R(d), *[P] * 9, BIG, None) == code and L.ax_matmul_q4_workspace_bytes(R(d)) == 0
    assert L.ax_gated_q4(R(d), *[P] * 9, BIG, None) == code and L.ax_gated_q4_workspace_bytes(R(d)) == 0


def test_4_bit_product_pointers():
    L, d = ax.lib(), q4()
    go = lambda *a: L.ax_matmul_q4(R(d), *a, P, BIG, None)  # noqa: E731
    null_each(go, 8, skip=(5, 6))
    odd_each(go, 8)
    copied = q4(unaligned=1, rows=2000, N=4096, y_ld=4096, residual_ld=4096)
    need = L.ax_matmul_q4_workspace_bytes(R(copied))
    assert need >= 2000 * 64 and L.ax_matmul_q4(R(copied), *[P] * 8, P, need - 1, None) == -5
    copied.unaligned = 0  # (rows found through the index, in place)
    assert L.ax_matmul_q4_workspace_bytes(R(copied)) == 0 and L.ax_matmul_q4_workspace_bytes(R(q4(rows=8, unaligned=1))) == 0
    assert L.ax_matmul_q4_workspace_bytes(R(q4(N=4096, y_ld=4096, residual_ld=4096))) >= 4 * 4096 * 64  # weights written out
    assert L.ax_matmul_q4(R(q4(residual_ld=3)), *[P] * 9, BIG, None) == -2
    gated = lambda *a: L.ax_gated_q4(R(d), *a, P, BIG, None)  # noqa: E731
    null_each(gated, 8)
    odd_each(gated, 8)
    assert L.ax_matmul_q4(R(q4(rows=0)), *[None] * 9, 0, None) == 0


def test_python_side():
    x, w, o = torch.ones((4, 8)), torch.ones((2, 8, 8)), torch.zeros(3, dtype=torch.int32)
    rows = torch.zeros((4, 2), dtype=torch.int32)
    for call in (lambda: ax.ax_route(x, 2), lambda: ax.ax_route_backward(x, x, rows, x), lambda: ax.ax_matmul_experts(x, w, o),
                 lambda: ax.ax_gated_experts(x, w, w, o), lambda: ax.ax_matmul_experts_backward(x, x, w, o),
                 lambda: ax.ax_gated_experts_backward(x, x, w, w, x, x, o), lambda: ax.ax_combine(x, rows), lambda: ax.ax_combine_backward(x, x, rows),
                 lambda: ax.ax_quantize_q4(x), lambda: ax.ax_pack_q4(x.to(torch.int8), x.to(torch.bfloat16)), lambda: ax.ax_matmul_q4(x, x),
                 lambda: ax.ax_gated_q4(x, x, x)):
        with pytest.raises(TypeError):  # not on the GPU, or not of the type: no fallback
            call()


def test_more_tiles_than_a_launch_has():
    L, many = ax.lib(), dict(rows=1 << 30, x_rows=1 << 30, N=1, K=1, x_ld=1, y_ld=1, dtype=0, indexed=0)
    d = experts(w_ld=1, gx_ld=1, **many)
    assert L.ax_matmul_experts(R(d), P, None, P, P, P, None, P, BIG, None) == -2
    assert L.ax_gated_experts(R(d), P, None, P, P, P, P, None, None, P, BIG, None) == -2
    assert L.ax_matmul_experts_backward(R(d), P, P, None, P, P, None, P, P, P, BIG, None) == -2
    assert L.ax_gated_experts_backward(R(d), P, P, None, P, P, P, P, P, P, P, P, P, BIG, None) == -2
    assert L.ax_matmul_q4(R(q4(residual_ld=1, **many)), P, None, P, P, P, None, None, P, P, BIG, None) == -2
    assert L.ax_gated_q4(R(q4(residual_ld=1, **many)), P, None, P, P, P, P, P, P, P, BIG, None) == -2
