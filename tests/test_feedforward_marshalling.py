"""What the feed-forward entry points hand to the library, on the host: the C calls are replaced by ones that take notes, and the
tensors are ordinary ones that say that they are on the GPU."""

import contextlib

import pytest
import torch

from paper_2002_09481_amd import binding as ax
from paper_2002_09481_amd.feedforward import FeedForward


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


class Side:
    """A stream that is not the current one, for tensors on the host."""

    device, cuda_stream = torch.device("cuda", 0), 7


def _every_operator():
    """(call, its arguments in their order) of every operator that allocates."""
    f = lambda *s: floats(*s, dtype=torch.float32)  # noqa: E731
    q, sc = codes(4, 16), f(4)
    x, w, gy, v = f(4, 16), f(16, 16), f(4, 16), f(16)
    opt = ax.AxAdamW([v], [f(16)], [codes(16)], [placed(torch.zeros(16, dtype=torch.uint8))], [f(1)], [f(1)])
    return [(ax.ax_rmsnorm, (x, v, gy)), (ax.ax_rmsnorm_q8, (x, v, gy, 1e-5, True, None, None, None, None, True)),
            (ax.ax_rmsnorm_backward, (gy, x, v, sc)), (ax.ax_matmul, (x, w, v, gy, "silu", False, None, True)),
            (ax.ax_matmul_q8, (q, sc, q, sc)), (ax.ax_matmul_backward, (gy, x, w)), (ax.ax_gated, (x, w, w, "silu", None, True)),
            (ax.ax_gated_q8, (q, sc, q, sc, q, sc)), (ax.ax_gated_backward, (gy, x, w, w, gy, gy)), (opt.states, ())]


class Streams:
    """The current stream (a stack), and who allocated and tied what: made holds (address, current stream then), ties (address,
    stream)."""

    def __init__(self, monkeypatch):
        self.main, self.side, self.made, self.ties = object(), Side(), [], []
        self.current = [self.main]

        @contextlib.contextmanager
        def on(s):
            self.current.append(s)
            try:
                yield
            finally:
                self.current.pop()

        def factory(f):
            def make(*a, **kw):
                t = placed(f(*a, **{n: v for n, v in kw.items() if n != "device"}))
                self.made.append((t.data_ptr(), self.current[-1]))
                return t
            return make

        monkeypatch.setattr(torch.cuda, "stream", on)
        monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: self.current[-1])
        monkeypatch.setattr(Placed, "record_stream", lambda t, s: self.ties.append((t.data_ptr(), s)), raising=False)
        for name in ("empty", "empty_like", "empty_strided"):
            monkeypatch.setattr(torch, name, factory(getattr(torch, name)))
        monkeypatch.setattr(Placed, "new_empty", factory(torch.Tensor.new_empty), raising=False)

    def check(self, call, args):
        """What a call allocates belongs to its stream's pool; what it takes is tied to its stream, what it returns to the one
        that was current."""
        out = call(*args, stream=self.side)
        results = [t for t in (out if isinstance(out, tuple) else (out,)) if isinstance(t, torch.Tensor)]
        results += [ts[0] for ts in out if isinstance(ts, list)] if isinstance(out, tuple) else []
        assert self.made and results and all(where is self.side for _, where in self.made) and self.current == [self.main]
        assert all((t.data_ptr(), self.main) in self.ties for t in results)
        assert all((t.data_ptr(), self.side) in self.ties for t in args if isinstance(t, torch.Tensor))


@pytest.mark.parametrize("k", range(10))
def test_memory_of_calls_on_another_stream(notes, monkeypatch, k):
    call, args = _every_operator()[k]
    Streams(monkeypatch).check(call, args)
    assert len(notes.calls) == 1


def test_gradients_of_a_step_on_another_stream(notes, monkeypatch):
    ties, side = [], Side()
    monkeypatch.setattr(Placed, "record_stream", lambda t, s: ties.append((t.data_ptr(), s)), raising=False)
    p, g, factor = (floats(n, dtype=torch.float32) for n in (16, 16, 1))
    opt = ax.AxAdamW([p], [g], m=[floats(16, dtype=torch.float32)], v=[floats(16, dtype=torch.float32)])
    opt.step(1e-3, 1, grad_scale=factor)
    assert not ties
    opt.step(1e-3, 2, grad_scale=factor, stream=side)
    assert (g.data_ptr(), side) in ties and (factor.data_ptr(), side) in ties


def _kept_block():
    f = lambda *s: floats(*s, dtype=torch.float32)  # noqa: E731
    b = FeedForward.__new__(FeedForward)
    b.width, b.hidden, b.act, b.dtype, b.eps = 16, 24, "silu", torch.float32, 1e-5
    b.params = {"wg": f(16, 24), "wu": f(16, 24), "wd": f(24, 16), "norm": f(16), "bias": f(16)}
    b.grads = {n: torch.zeros_like(t) for n, t in b.params.items()}
    b._kept = (f(4, 16), f(4, 16), f(4), f(4, 24), f(4, 24), f(4, 24))
    return b


@pytest.mark.parametrize("way", ["argument", "current"])
def test_what_a_backward_pass_on_another_stream_drops(notes, monkeypatch, way):
    """The forward pass left it in another stream's pool: it is tied to the stream that reads it before it dies."""
    b, gy, s = _kept_block(), floats(4, 16, dtype=torch.float32), Streams(monkeypatch)
    kept = [t.data_ptr() for t in b._kept]
    if way == "argument":
        gx = b.backward(gy, stream=s.side)
        assert (gx.data_ptr(), s.main) in s.ties
    else:
        with torch.cuda.stream(s.side):
            b.backward(gy)
    assert b._kept is None and all((k, s.side) in s.ties for k in kept)
    assert notes.calls == ["ax_matmul_backward", "ax_gated_backward", "ax_rmsnorm_backward"]


def test_results_of_a_block_on_another_stream(notes, monkeypatch):
    b, s = _kept_block(), Streams(monkeypatch)
    x, r = floats(4, 16, dtype=torch.float32), floats(4, 16, dtype=torch.float32)
    s.check(b.forward, (x, r))


def test_a_call_on_another_stream_that_fails(notes, monkeypatch):
    """Its operands are tied to the stream all the same, and the current stream is the one that it was."""
    s = Streams(monkeypatch)
    x, w = floats(4, 16, dtype=torch.float32), floats(16, 16, dtype=torch.float32)
    notes.ax_matmul = lambda *a: -6
    monkeypatch.setattr(ax, "_check", lambda rc: (_ for _ in ()).throw(ax.AxError(rc, "")) if rc else None)
    with pytest.raises(ax.AxError):
        ax.ax_matmul(x, w, stream=s.side)
    assert s.current == [s.main] and (x.data_ptr(), s.side) in s.ties and (w.data_ptr(), s.side) in s.ties
    with pytest.raises(TypeError):  # nothing on the host is tied to a stream (other sizes: those above are known as checked)
        ax.ax_matmul(torch.zeros((5, 16)), w, stream=s.side)
