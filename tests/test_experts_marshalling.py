"""What the entry points of a block of experts hand to the library, on the host: shapes, types and places that they refuse, memory of
calls on another stream."""

import pytest
import torch

from paper_2002_09481_amd import binding as ax
from paper_2002_09481_amd.feedforward import ExpertsFeedForward
from test_feedforward_marshalling import Notes, Placed, Streams, floats, placed


class Sizes(Notes):
    def ax_q4_codes_bytes(self, *a):
        return 1024

    def ax_q4_scales_bytes(self, *a):
        return 64


@pytest.fixture
def notes(monkeypatch):
    n = Sizes()
    monkeypatch.setattr(ax, "lib", lambda: n)
    monkeypatch.setattr(ax, "_stream_ptr", lambda s: 0)
    monkeypatch.setattr(ax, "_checked", {})
    return n


f32 = lambda *s: floats(*s, dtype=torch.float32)  # noqa: E731
whole = lambda *s: placed(torch.zeros(s, dtype=torch.int32))  # noqa: E731


def weights4(experts=None, rows=16, cols=16, group=32):
    w = ax.AxQ4(rows, cols, group, experts, "cpu")
    w.codes, w.scales = placed(w.codes), placed(w.scales)
    return w


def _operators():
    """(call, its arguments in their order, the C functions it ends in) of every operator."""
    x, l, w, o, t = f32(6, 16), f32(6, 3), f32(3, 16, 16), whole(4), whole(12)
    y, rows, p = f32(12, 16), whole(6, 2), f32(6, 2)
    return [(ax.ax_route, (l, 2), "ax_route"), (ax.ax_route_backward, (p, l, rows, p), "ax_route_backward"),
            (ax.ax_matmul_experts, (x, w, o, t, "silu", False, True), "ax_matmul_experts"),
            (ax.ax_matmul_experts_backward, (y, x, w, o, t), "ax_matmul_experts_backward"),
            (ax.ax_gated_experts, (x, w, w, o, t, "silu", True), "ax_gated_experts"),
            (ax.ax_gated_experts_backward, (y, x, w, w, y, y, o, t), "ax_gated_experts_backward"),
            (ax.ax_combine, (y, rows, p, x), "ax_combine"), (ax.ax_combine_backward, (x, y, rows, p), "ax_combine_backward"),
            (ax.ax_quantize_q4, (w,), "ax_quantize_q4"),
            (ax.ax_pack_q4, (placed(torch.zeros((16, 16), dtype=torch.int8)), floats(16, 1)), "ax_pack_q4"),
            (ax.ax_matmul_q4, (x, weights4(3), None, None, "none", o, t), "ax_matmul_q4"),
            (ax.ax_gated_q4, (x, weights4(3), weights4(3), "silu", o, t), "ax_gated_q4")]


@pytest.mark.parametrize("k", range(12))
def test_memory_of_calls_on_another_stream(notes, monkeypatch, k):
    call, args, name = _operators()[k]
    s = Streams(monkeypatch)
    out = call(*args, stream=s.side)
    results = list(ax._tensors_of(out if isinstance(out, tuple) else (out,)))
    assert s.made and results and all(where is s.side for _, where in s.made) and s.current == [s.main]
    assert all((t.data_ptr(), s.main) in s.ties for t in results)
    assert all((t.data_ptr(), s.side) in s.ties for t in ax._tensors_of(args))
    assert notes.calls == [name]


def test_values_of_4_bit_weights_on_another_stream(notes, monkeypatch):
    w, s = weights4(), Streams(monkeypatch)
    out = w.values(stream=s.side)
    assert out.shape == (16, 16) and all((t.data_ptr(), s.side) in s.ties for t in (w.codes, w.scales)) and (out.data_ptr(), s.main) in s.ties


@pytest.mark.parametrize("k", range(12))
def test_other_float_types(notes, k):
    call, args, _ = _operators()[k]
    for dtype in (torch.float16, torch.float64):
        bad = [placed(a.to(dtype)) if isinstance(a, torch.Tensor) and a.is_floating_point() else a for a in args]
        with pytest.raises((TypeError, ValueError)):
            call(*bad)
    assert not notes.calls


@pytest.mark.parametrize("k", [0, 1, 2, 3, 4, 5, 6, 7, 10, 11])
def test_whole_numbers_are_32_bits_wide(notes, k):
    call, args, _ = _operators()[k]
    bad = [placed(a.long()) if isinstance(a, torch.Tensor) and a.dtype == torch.int32 else a for a in args]
    if any(a is not b for a, b in zip(args, bad)):
        with pytest.raises(TypeError):
            call(*bad)
    assert not notes.calls


def test_shapes(notes):
    x, w, o, t = f32(6, 16), f32(3, 16, 24), whole(4), whole(12)
    y, rows = f32(12, 24), whole(6, 2)
    for call in (lambda: ax.ax_route(f32(6, 3), 4), lambda: ax.ax_route(f32(6, 3), 0), lambda: ax.ax_route(f32(6, 3), 2, rows_out=whole(6, 3)),
                 lambda: ax.ax_route_backward(f32(6, 3), f32(6, 3), rows, f32(6, 2)),
                 lambda: ax.ax_matmul_experts(x, w, whole(3)), lambda: ax.ax_matmul_experts(x, f32(16, 24), o), lambda: ax.ax_matmul_experts(f32(6, 8), w, o),
                 lambda: ax.ax_matmul_experts(x, w, o, transposed=True), lambda: ax.ax_matmul_experts(x, w, o, t, y_out=f32(6, 24)),
                 lambda: ax.ax_matmul_experts(x, placed(torch.zeros((3, 32, 24)))[:, :16], o), lambda: ax.ax_matmul_experts(x, w, o, act="tanh"),
                 lambda: ax.ax_gated_experts(x, w, f32(3, 16, 16), o), lambda: ax.ax_gated_experts_backward(y, x, w, w, y, f32(11, 24), o, t),
                 lambda: ax.ax_matmul_experts_backward(y, x, w, o, t, act="silu"), lambda: ax.ax_matmul_experts_backward(f32(6, 24), x, w, o, t),
                 lambda: ax.ax_matmul_experts_backward(y, x, w, o, t, gw_out=f32(3, 24, 16)),
                 lambda: ax.ax_combine(y, whole(12)), lambda: ax.ax_combine(y, rows, f32(6, 3)), lambda: ax.ax_combine(y, rows, residual=f32(5, 24)),
                 lambda: ax.ax_combine_backward(f32(5, 24), y, rows), lambda: ax.ax_combine_backward(f32(6, 24), y, rows, gh_out=f32(11, 24)),
                 lambda: ax.ax_quantize_q4(f32(4, 8), group=16), lambda: ax.ax_quantize_q4(f32(2, 2, 4, 8)),
                 lambda: ax.ax_pack_q4(placed(torch.zeros((4, 40), dtype=torch.int8)), floats(4, 1), group=32),
                 lambda: ax.ax_matmul_q4(f32(4, 8), weights4()), lambda: ax.ax_matmul_q4(x, weights4(3)), lambda: ax.ax_matmul_q4(x, weights4(), bias=f32(8)),
                 lambda: ax.ax_matmul_q4(x, weights4(3), offsets=whole(3)), lambda: ax.ax_gated_q4(x, weights4(), weights4(group=64)),
                 lambda: ax.ax_gated_q4(x, weights4(), weights4(rows=8))):
        with pytest.raises(ValueError):
            call()
    assert not notes.calls


def test_shapes_of_results(notes):
    x, o, t = f32(6, 16), whole(4), whole(12)
    e, w, off, rows, tok = ax.ax_route(f32(2, 3, 5), 2)
    assert e.shape == w.shape == rows.shape == (2, 3, 2) and off.shape == (6,) and tok.shape == (12,)
    assert ax.ax_matmul_experts(x, f32(3, 16, 24), o)[0].shape == (6, 24) and ax.ax_matmul_experts(x, f32(3, 24, 16), o, t, transposed=True)[0].shape == (12, 24)
    gx, gw = ax.ax_matmul_experts_backward(f32(12, 24), x, f32(3, 16, 24), o, t)
    assert gx.shape == (12, 16) and gw.shape == (3, 16, 24)
    assert ax.ax_combine(f32(12, 24), whole(2, 3, 2)).shape == (2, 3, 24)
    assert ax.ax_matmul_q4(f32(2, 3, 16), weights4()).shape == (2, 3, 16) and ax.ax_gated_q4(x, weights4(3), weights4(3), offsets=o, tokens=t).shape == (12, 16)
    wide = placed(torch.zeros((3, 16, 40)))[..., :24]
    gx, gw = ax.ax_matmul_experts_backward(f32(12, 24), x, wide, o, t)
    assert gw.stride() == wide.stride()


def test_tensors_on_other_devices(notes, monkeypatch):
    """Tensors of two devices, or of one that is not the current one, never reach the library."""

    class Elsewhere(Placed):
        device = torch.device("cuda", 1)

    far = lambda t: t.as_subclass(Elsewhere)  # noqa: E731
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    for call, args, name in _operators():
        places = [i for i, a in enumerate(args) if isinstance(a, torch.Tensor)]
        for i in places:
            if name in ("ax_quantize_q4",) or len(places) == 1:
                continue
            with pytest.raises(ValueError):
                call(*[far(a) if j == i else a for j, a in enumerate(args)])
        with pytest.raises(ValueError):
            call(*[far(a) if isinstance(a, torch.Tensor) else a for a in args])
    assert not notes.calls


def test_what_a_backward_pass_on_another_stream_drops(notes, monkeypatch):
    b = ExpertsFeedForward.__new__(ExpertsFeedForward)
    b.width, b.hidden, b.experts, b.k, b.act, b.dtype, b.eps, b.normalize = 16, 24, 3, 2, "silu", torch.float32, 1e-5, True
    b.params = {"router": f32(16, 3), "wg": f32(3, 16, 24), "wu": f32(3, 16, 24), "wd": f32(3, 24, 16), "norm": f32(16)}
    b.grads = {n: placed(torch.zeros_like(t)) for n, t in b.params.items()}
    b._kept = (f32(4, 16), f32(4, 16), f32(4), f32(4, 3), whole(4, 2), f32(4, 2), whole(4), whole(4, 2), whole(8), f32(8, 24), f32(8, 24), f32(8, 24),
               f32(8, 16))
    kept = [t.data_ptr() for t in b._kept]
    s = Streams(monkeypatch)
    gx = b.backward(f32(4, 16), stream=s.side)
    assert b._kept is None and all((k, s.side) in s.ties for k in kept) and (gx.data_ptr(), s.main) in s.ties
    assert notes.calls == ["ax_combine_backward", "ax_matmul_experts_backward", "ax_gated_experts_backward", "ax_route_backward", "ax_matmul_backward",
                           "ax_combine", "ax_rmsnorm_backward"]
