"""What the lookup entry points allocate for calls on another stream, on the host: the C calls are replaced by ones that take notes."""

import os

import pytest
import torch

from paper_2002_09481_amd import binding as ax
from test_feedforward_marshalling import Streams, floats, notes, placed  # noqa: F401



def _calls():
    u8 = lambda *s: placed(torch.zeros(s, dtype=torch.uint8))  # noqa: E731
    f = lambda *s: floats(*s, dtype=torch.float32)  # noqa: E731
    lut, luts = placed(torch.zeros(65536, dtype=torch.int16)), placed(torch.zeros((2, 65536), dtype=torch.int16))

    class q:
        x_scale, x_zp, w_scale, w_zp, pad_code = 1.0, 0, 1.0, 0, None

    x, w, xf, wf = u8(1, 6, 6, 4), u8(3, 3, 4, 8), f(1, 6, 6, 4), f(3, 3, 4, 8)
    return [(ax.ax_conv2d, (x, w, lut, 1, 1, q)), (ax.ax_dense, (u8(3, 8), u8(8, 5), lut, q)),
            (ax.ax_conv2d_multi_lut, (x, w, luts, 1, 1, q)), (ax.ax_conv2d_ex, (x, w, lut, 1, 1, q)),
            (ax.ax_conv2d_transpose, (x, w, lut, 1, 0, q)), (ax.ax_conv2d_backward, (x, w, f(1, 6, 6, 8), 1, 1, q)),
            (ax.ax_range_f32, (xf,)), (ax.ax_quantize_f32, (xf, f(2))), (ax.ax_conv2d_f32, (xf, wf, lut, 1, 1)),
            (ax.ax_conv2d_f32_ex, (xf, wf, lut, 1, 1)), (ax.ax_dense_f32, (f(3, 8), f(8, 5), lut))]


@pytest.mark.parametrize("k", range(11))
def test_memory_of_calls_on_another_stream(notes, monkeypatch, k):  # noqa: F811
    call, args = _calls()[k]
    Streams(monkeypatch).check(call, args)


@pytest.mark.skipif(not os.path.exists(ax.LIB_PATH), reason="libaxconv.so not built")
def test_a_layers_own_workspace_on_another_stream(monkeypatch):
    """Allocated in the pool of the first stream that runs the layer, tied to each one that does."""
    f = lambda *s: placed(torch.zeros(s, dtype=torch.uint8))  # noqa: E731
    d = ax.ax_conv_desc_t(1, 8, 8, 16, 3, 3, 16, 1, 1, 1, 1, 1, 1, 0, 0)
    with ax.AxLayer(d, ax.ax_quant_t(1.0, 0, 1.0, 0, -1)) as layer:
        s = Streams(monkeypatch)
        monkeypatch.setattr(ax, "_check", lambda rc: None)
        monkeypatch.setattr(ax, "_stream_ptr", lambda stream: 0)
        real = ax.lib()

        class Stub:
            def __getattr__(self, name):
                return (lambda *a: 0) if name in ("ax_layer_run", "ax_layer_prepare") else getattr(real, name)

        stub = Stub()
        monkeypatch.setattr(ax, "lib", lambda: stub)
        s.check(layer.prepare, (f(3, 3, 16, 16), placed(torch.zeros(65536, dtype=torch.int16))))
        s.check(layer.run, (f(1, 8, 8, 16),))
        assert (layer._ws.data_ptr(), s.side) in s.made and (layer._ws.data_ptr(), s.side) in s.ties
        monkeypatch.setattr(ax, "lib", lambda: real)
