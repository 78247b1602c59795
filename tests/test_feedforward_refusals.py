"""What the feed-forward entry points refuse, on the host, before any device work."""

import ctypes
import os

import pytest
import torch

from paper_2002_09481_amd import binding as ax

pytestmark = pytest.mark.skipif(not os.path.exists(ax.LIB_PATH), reason="libaxconv.so not built")
P, ODD = ctypes.c_void_p(4096), ctypes.c_void_p(4097)
R = ctypes.byref


def norm(**kw):
    d = ax.ax_norm_desc_t(4, 64, 64, 64, 64, 64, 1, 1, 1e-5, 1)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def mm(**kw):
    d = ax.ax_matmul_desc_t(4, 64, 32, 32, 64, 64, 64, 1, 1, 0, 0, 0)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("bad,code", [(dict(rows=-1), -2), (dict(cols=0), -2), (dict(x_ld=63), -2), (dict(y_ld=10), -2),
                                      (dict(residual_ld=1), -2), (dict(sum_ld=0), -2), (dict(dtype=2), -8), (dict(w_dtype=-1), -8),
                                      (dict(eps=-1.0), -8), (dict(eps=float("nan")), -8), (dict(normalize=2), -8), (dict(normalize=0), -8)])
def test_norm_descriptions(bad, code):
    assert ax.lib().ax_rmsnorm(R(norm(**bad)), P, P, P, P, P, P, None) == code


def test_norm_pointers():
    L, d = ax.lib(), norm()
    assert L.ax_rmsnorm(None, P, P, P, P, P, P, None) == -1
    for k in (0, 2, 4):  # x, weight, y
        args = [P] * 6
        args[k] = None
        assert L.ax_rmsnorm(R(d), *args, None) == -1
    assert L.ax_rmsnorm(R(d), P, None, P, P, P, P, None) == -1  # a sum without a residual
    for k in range(6):
        args = [P] * 6
        args[k] = ODD
        assert L.ax_rmsnorm(R(d), *args, None) == -7
    assert L.ax_rmsnorm_q8(R(d), P, P, P, P, None, P, P, None) == -1
    assert L.ax_rmsnorm_q8(R(d), P, P, P, P, P, None, P, None) == -1
    assert L.ax_rmsnorm_q8(R(d), P, P, P, P, P, ctypes.c_void_p(4098), P, None) == -7
    need = L.ax_rmsnorm_backward_workspace_bytes(R(d))
    assert need >= 256 and L.ax_rmsnorm_backward_workspace_bytes(R(norm(cols=0))) == 0
    back = lambda *a: L.ax_rmsnorm_backward(R(d), *a)  # noqa: E731
    assert back(P, P, P, P, P, None, None, P, need, None) == -1
    assert back(P, P, P, P, None, P, P, P, need, None) == -1
    assert back(P, P, P, P, P, P, P, P, need - 1, None) == -5
    assert back(P, P, P, P, P, P, P, None, need, None) == -5
    assert back(P, P, P, P, P, P, P, ctypes.c_void_p(4096 + 16), need, None) == -5
    assert L.ax_rmsnorm_backward(R(norm(normalize=0)), P, P, P, P, P, P, P, P, need, None) == -8


BAD = [(dict(M=-1), -2), (dict(N=0), -2), (dict(K=0), -2), (dict(M=1 << 31), -2), (dict(x_ld=31), -2), (dict(w_ld=63), -2),
       (dict(y_ld=63), -2), (dict(x_ld=1 << 21), -2), (dict(dtype=2), -8), (dict(out_dtype=5), -8), (dict(act=4), -8), (dict(act=-1), -8),
       (dict(w_transposed=2), -8), (dict(unaligned=-1), -8)]


@pytest.mark.parametrize("bad,code", BAD)
def test_product_descriptions(bad, code):
    L, d, ws = ax.lib(), mm(**bad), 1 << 30
    assert L.ax_matmul(R(d), P, P, P, P, P, P, P, ws, None) == code and L.ax_matmul_workspace_bytes(R(d)) == 0
    assert L.ax_matmul_backward(R(d), P, P, P, P, P, P, P, P, ws, None) == code and L.ax_matmul_backward_workspace_bytes(R(d)) == 0
    assert L.ax_gated(R(d), P, P, P, P, P, P, P, ws, None) == code and L.ax_gated_workspace_bytes(R(d)) == 0
    assert L.ax_gated_backward(R(d), P, P, P, P, P, P, P, P, P, P, ws, None) == code and L.ax_gated_backward_workspace_bytes(R(d)) == 0


def test_products_of_codes():
    L, ws = ax.lib(), 1 << 30
    q8 = lambda d, *a: L.ax_matmul_q8(R(d), *(a or [P] * 8), ws, None)  # noqa: E731
    g8 = lambda d: L.ax_gated_q8(R(d), *[P] * 8, ws, None)  # noqa: E731
    flat = dict(w_transposed=1, K=32, w_ld=32)
    assert q8(mm()) == -8 and g8(mm()) == -8  # codes are [N, K]
    assert q8(mm(w_transposed=1, K=131072, x_ld=131072, w_ld=131072)) == -4 and g8(mm(w_transposed=1, K=131072, x_ld=131072, w_ld=131072)) == -4
    assert q8(mm(**flat, residual_ld=3)) == -2
    for k in (0, 1, 2, 3, 6):  # x, its scales, w, its scales, y
        args = [P] * 8
        args[k] = None
        assert q8(mm(**flat), *args) == -1
    args = [P] * 8
    args[1] = ctypes.c_void_p(4098)
    assert q8(mm(**flat), *args) == -7
    args[1], args[0] = P, ctypes.c_void_p(4096 + 8)  # rows of whole 16-byte pieces have to start on one
    assert q8(mm(**flat), *args) == -7


def test_product_pointers():
    L = ax.lib()
    d = mm(M=72, dtype=0, out_dtype=0)  # float32 operands go through the workspace (of more than a few rows)
    need = L.ax_matmul_workspace_bytes(R(d))
    assert need >= 3 * 2 * (72 * 32 + 32 * 64)
    assert L.ax_matmul(R(d), P, P, P, P, P, P, P, need - 1, None) == -5 and L.ax_matmul(R(d), P, P, P, P, P, P, None, need, None) == -5
    assert L.ax_matmul(R(d), P, P, P, P, P, P, ctypes.c_void_p(4096 + 64), need, None) == -5
    assert L.ax_matmul(None, P, P, P, P, P, P, P, need, None) == -1
    for k in (0, 1, 4):  # x, w, y
        args = [P] * 6
        args[k] = None
        assert L.ax_matmul(R(d), *args, P, need, None) == -1
    for k in range(6):
        args = [P] * 6
        args[k] = ctypes.c_void_p(4098)
        assert L.ax_matmul(R(d), *args, P, need, None) == -7
    assert L.ax_matmul(R(mm()), ctypes.c_void_p(4098), P, P, P, P, P, P, need, None) == -7
    assert L.ax_matmul(R(mm(residual_ld=1)), P, P, P, P, P, P, P, need, None) == -2
    need = L.ax_matmul_backward_workspace_bytes(R(d))
    back = lambda d, *a: L.ax_matmul_backward(R(d), *a, P, need, None)  # noqa: E731
    assert back(d, P, P, P, P, None, None, None) == -1 and back(d, None, P, P, P, P, P, P) == -1
    assert back(d, P, None, P, P, P, P, P) == -1 and back(d, P, P, None, P, P, P, P) == -1
    assert back(mm(dtype=0, out_dtype=0, act=2), P, P, P, None, P, P, P) == -1
    assert back(mm(dtype=0, out_dtype=1), P, P, P, P, P, P, P) == -8
    assert L.ax_matmul_backward(R(d), P, P, P, P, P, P, P, P, need - 1, None) == -5
    gb = lambda *a: L.ax_gated_backward(R(d), *a, P, 1 << 30, None)  # noqa: E731
    assert gb(P, P, P, P, P, P, P, P, None) == -1 and gb(P, P, P, P, P, P, None, None, None) == -1 and gb(P, P, P, P, None, P, P, P, P) == -1
    assert L.ax_gated(R(d), P, P, P, P, P, None, P, 1 << 30, None) == -1  # one projection without the other
    assert L.ax_gated(R(mm(w_transposed=1, w_ld=32)), P, P, P, P, P, P, P, 1 << 30, None) == -8


def adam(**kw):
    d = ax.ax_adamw_desc_t(1e-3, 0.9, 0.999, 1e-8, 0.0, 1, None, 0, 0, 32, 0)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def tensor(**kw):
    t = (ax.ax_adamw_tensor_t * 1)(ax.ax_adamw_tensor_t(4096, 4096, 4096, 4096, 4096, 4096, None, 10))
    for k, v in kw.items():
        setattr(t[0], k, v)
    return t


@pytest.mark.parametrize("bad", [dict(step=0), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=float("nan")),
                                 dict(lr=float("inf")), dict(eps=-1.0), dict(weight_decay=float("nan")), dict(p_dtype=2), dict(g_dtype=-1),
                                 dict(state_bits=16), dict(reserved=1)])
def test_step_descriptions(bad):
    assert ax.lib().ax_adamw(R(adam(**bad)), tensor(), 1, None) == -8


def test_step_tensors():
    L = ax.lib()
    assert L.ax_adamw(None, tensor(), 1, None) == -1 and L.ax_adamw(R(adam()), None, 1, None) == -1
    assert L.ax_adamw(R(adam()), tensor(), -1, None) == -2 and L.ax_adamw(R(adam()), tensor(n=-1), 1, None) == -2
    for f in ("p", "g", "m", "v"):
        assert L.ax_adamw(R(adam()), tensor(**{f: None}), 1, None) == -1
        assert L.ax_adamw(R(adam()), tensor(**{f: 4098}), 1, None) == -7
    for f in ("m_scale", "v_scale"):
        assert L.ax_adamw(R(adam(state_bits=8)), tensor(**{f: None}), 1, None) == -1
        assert L.ax_adamw(R(adam(state_bits=8)), tensor(**{f: 4098}), 1, None) == -7
    assert L.ax_adamw(R(adam()), tensor(copy=4097), 1, None) == -7
    assert L.ax_adamw(R(adam(grad_scale=4097)), tensor(), 1, None) == -7
    assert L.ax_adamw(R(adam()), None, 0, None) == 0  # nothing to do
    assert L.ax_adamw(R(adam()), (ax.ax_adamw_tensor_t * 2)(), 2, None) == 0  # empty tensors need no memory
    out = (ctypes.c_void_p * 1)(4096)
    assert L.ax_adamw_states(tensor(), 1, None, out, None) == -1 and L.ax_adamw_states(tensor(m_scale=None), 1, out, out, None) == -1
    assert L.ax_adamw_states(tensor(), 1, out, (ctypes.c_void_p * 1)(4098), None) == -7 and L.ax_adamw_states(None, 0, None, None, None) == 0


def test_python_side():
    x, w = torch.ones((4, 8)), torch.ones((8, 8))
    for call in (lambda: ax.ax_rmsnorm(x, w[0]), lambda: ax.ax_matmul(x, w), lambda: ax.ax_gated(x, w, w),
                 lambda: ax.ax_rmsnorm_q8(x, w[0]), lambda: ax.ax_matmul_backward(x, x, w), lambda: ax.AxAdamW([x], [x])):
        with pytest.raises(TypeError):  # not on the GPU: no fallback
            call()
    with pytest.raises(ValueError):
        ax.AxAdamW([], [])
    with pytest.raises(ValueError):
        ax._act_code("tanh")
