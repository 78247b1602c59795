"""What objects hold and use on another stream than the current one, on the host: it is tied to that stream, since the object may be
dropped with the work under way."""

import pytest
import torch

from paper_2002_09481_amd import binding as ax
from paper_2002_09481_amd.feedforward import ExpertsFeedForward, FeedForward, QuantizedExperts, QuantizedFeedForward
from test_experts_marshalling import f32, notes, weights4, whole  # noqa: F401
from test_feedforward_marshalling import Streams, codes, placed


def _block(cls, weights, kept=()):
    b = cls.__new__(cls)
    b.act, b.dtype, b.eps, b.k, b.normalize, b._kept = "silu", torch.float32, 1e-5, 2, True, kept
    b.params = {n: f32(*s) for n, s in weights.items()}
    b.grads = {n: f32(*s) for n, s in weights.items()}
    return b


def _plain():
    return _block(FeedForward, {"wg": (16, 24), "wu": (16, 24), "wd": (24, 16), "norm": (16,), "bias": (16,)},
                  (f32(4, 16), f32(4, 16), f32(4), f32(4, 24), f32(4, 24), f32(4, 24)))


def _experts():
    return _block(ExpertsFeedForward, {"router": (16, 3), "wg": (3, 16, 24), "wu": (3, 16, 24), "wd": (3, 24, 16), "norm": (16,)},
                  (f32(4, 16), f32(4, 16), f32(4), f32(4, 3), whole(4, 2), f32(4, 2), whole(4), whole(4, 2), whole(8), f32(8, 24), f32(8, 24),
                   f32(8, 24), f32(8, 16)))


def _served(kind):
    b = (QuantizedExperts if kind == "experts" else QuantizedFeedForward).__new__(QuantizedExperts if kind == "experts" else QuantizedFeedForward)
    b.act, b.eps, b.dtype, b.k, b.normalize, b.norm = "silu", 1e-5, torch.float32, 2, True, f32(16)
    if kind == "experts":
        b.router, b.w = f32(16, 3), {"wg": weights4(3), "wu": weights4(3), "wd": weights4(3)}
        return b, [b.norm, b.router]
    b.bits, b.bias = kind, f32(16)
    b.w = {n: weights4() if kind == 4 else (codes(16, 16), f32(16)) for n in ("wg", "wu", "wd")}
    return b, [b.norm, b.bias]


def _tied(s, tensors):
    return all((t.data_ptr(), s.side) in s.ties for t in tensors)


@pytest.mark.parametrize("make", [_plain, _experts])
def test_parameters_and_gradients_of_a_block(notes, monkeypatch, make):  # noqa: F811
    b, s = make(), Streams(monkeypatch)
    b.forward(f32(4, 16), stream=s.side)
    assert _tied(s, b.params.values()) and not _tied(s, b.grads.values())
    s.ties.clear()
    b.backward(f32(4, 16), stream=s.side)
    assert _tied(s, b.params.values()) and _tied(s, b.grads.values())


@pytest.mark.parametrize("kind", [8, 4, "experts"])
def test_weights_of_a_served_block(notes, monkeypatch, kind):  # noqa: F811
    (b, vectors), s = _served(kind), Streams(monkeypatch)
    b.forward(f32(4, 16), stream=s.side)
    held = [t for w in b.w.values() for t in ((w.codes, w.scales) if isinstance(w, ax.AxQ4) else w)]
    assert len(held) == 6 and _tied(s, vectors + held)


@pytest.mark.parametrize("kind", [8, 4, "experts"])
def test_weights_laid_out_on_another_stream(notes, monkeypatch, kind):  # noqa: F811
    """What is read belongs to the block, what is made to whoever uses it next."""
    b = _experts() if kind == "experts" else _plain()
    b.master = {n: f32(*t.shape) for n, t in b.params.items()}
    s = Streams(monkeypatch)
    q = b.quantized(stream=s.side) if kind == "experts" else b.quantized(stream=s.side, bits=kind)
    assert _tied(s, [b.master[n] for n in ("wg", "wu", "wd")] + [b.params[n] for n in (("norm", "router") if kind == "experts" else ("norm", "bias"))])
    made = [q.norm, q.router if kind == "experts" else q.bias]
    made += [t for w in q.w.values() for t in ((w.codes, w.scales) if isinstance(w, ax.AxQ4) else w)]
    assert len(made) == 8 and all((t.data_ptr(), s.main) in s.ties for t in made) and s.current == [s.main]


@pytest.mark.parametrize("bits", [32, 8])
def test_parameters_and_states_of_an_optimizer(notes, monkeypatch, bits):  # noqa: F811
    """A step's are tied when the optimizer, which holds them, is dropped; those that states() reads in the call."""
    p, g, copy = f32(16), f32(16), placed(torch.zeros(16, dtype=torch.bfloat16))
    m, v = (codes(16), placed(torch.zeros(16, dtype=torch.uint8))) if bits == 8 else (f32(16), f32(16))
    scales = [f32(1), f32(1)] if bits == 8 else []
    opt = ax.AxAdamW([p], [g], [m], [v], *([t] for t in scales), copies=[copy])
    s = Streams(monkeypatch)
    if bits == 8:
        opt.states(stream=s.side)
        assert _tied(s, [m, v] + scales)
        s.ties.clear()
    opt.step(1e-3, 1, stream=s.side)
    opt.step(1e-3, 2)
    assert _tied(s, [g])
    del opt
    assert _tied(s, [p, m, v, copy] + scales) and not [t for t, where in s.ties if where is not s.side]
    s.ties.clear()
    opt = ax.AxAdamW([p], [g], [m], [v], *([t] for t in scales), copies=[copy])
    opt.step(1e-3, 1)
    del opt
    assert not s.ties


def test_what_a_lookup_layer_was_prepared_from(notes, monkeypatch):  # noqa: F811
    """Filters, tables and the prepared block are tied to each stream that runs the layer, its workspace to the current one too."""
    u8 = lambda *s: placed(torch.zeros(s, dtype=torch.uint8))  # noqa: E731
    w, luts, x, acc, y = u8(3, 3, 16, 16), placed(torch.zeros(65536, dtype=torch.int16)), u8(1, 8, 8, 16), whole(1, 8, 8, 16), f32(1, 8, 8, 16)
    layer = ax.AxLayer(ax.ax_conv_desc_t(1, 8, 8, 16, 3, 3, 16, 1, 1, 1, 1, 1, 1, 0, 0), ax.ax_quant_t(1.0, 0, 1.0, 0, -1))
    prepared = placed(layer.prepare(w, luts, prepared=u8(512)))
    s = Streams(monkeypatch)
    for call in (lambda: layer.run(x, stream=s.side), lambda: layer.run_static(x, acc, y, stream=s.side), lambda: layer.kernel_ms(x, stream=s.side)):
        s.ties.clear()
        call()
        assert _tied(s, [w, luts, prepared])
    layer.run(x, stream=s.side)
    assert _tied(s, [layer._ws]) and (layer._ws.data_ptr(), s.main) in s.ties
