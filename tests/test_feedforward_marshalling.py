"""What the feed-forward entry points hand to the library, on the host: the C calls are replaced by ones that take notes, and the
tensors are ordinary ones that say that they are on the GPU."""

import pytest
import torch

from paper_2002_09481_amd import binding as ax


class Placed(torch.Tensor):
    is_cuda = True


def placed(t):
    return t.as_subclass(Placed)


class Notes:
    """Stands for the library: workspace queries give `need` bytes, every other call succeeds; calls holds their names."""

    def __init__(self, need=512):
        self.calls, self.need = [], need

    def __getattr__(self, name):
        if name.endswith("_workspace_bytes"):
            return lambda *a: self.need

        def call(*a):
            self.calls.append(name)
            return 0

        return call


@pytest.fixture
def notes(monkeypatch):
    n = Notes()
    monkeypatch.setattr(ax, "lib", lambda: n)
    monkeypatch.setattr(ax, "_stream_ptr", lambda s: 0)
    monkeypatch.setattr(ax, "_checked", {})
    return n


def codes(*shape):
    return placed(torch.zeros(shape, dtype=torch.int8))


def floats(*shape, dtype=torch.bfloat16):
    return placed(torch.zeros(shape, dtype=dtype))


@pytest.mark.parametrize("out", [None, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dtype", [torch.int8, torch.uint8, torch.float16, torch.float64, torch.int32])
def test_float_products_take_float_operands_alone(notes, dtype, out):
    x, w = (placed(torch.zeros((4, 16), dtype=dtype)) for _ in range(2))
    y = floats(4, 4)
    for call in (lambda: ax.ax_matmul(x, w, transposed=True, out_dtype=out), lambda: ax.ax_matmul(x, placed(w.t().contiguous()), out_dtype=out),
                 lambda: ax.ax_gated(x, placed(w.t().contiguous()), placed(w.t().contiguous()), out_dtype=out),
                 lambda: ax.ax_matmul_backward(y, x, w, transposed=True), lambda: ax.ax_gated_backward(y, x, placed(w.t().contiguous()),
                                                                                                    placed(w.t().contiguous()), y, y)):
        with pytest.raises(TypeError):
            call()
    assert not notes.calls


def test_products_of_codes_take_codes_alone(notes):
    x, w, s, s16 = floats(4, 16), floats(8, 16), floats(4, dtype=torch.float32), floats(8, dtype=torch.float32)
    for a, b in ((x, w), (codes(4, 16), w), (x, codes(8, 16))):
        with pytest.raises(TypeError):
            ax.ax_matmul_q8(a, s, b, s16)
        with pytest.raises(TypeError):
            ax.ax_gated_q8(a, s, b, s16, b, s16)
    with pytest.raises(TypeError):
        ax.ax_gated_q8(codes(4, 16), s, codes(8, 16), s16, w, s16)
    assert not notes.calls
    ax.ax_matmul_q8(codes(4, 16), s, codes(8, 16), s16)
    ax.ax_gated_q8(codes(4, 16), s, codes(8, 16), s16, codes(8, 16), s16)
    ax.ax_matmul(x, w, transposed=True)
    assert notes.calls == ["ax_matmul_q8", "ax_gated_q8", "ax_matmul"]
