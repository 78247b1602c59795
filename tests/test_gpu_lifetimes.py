"""Objects that are dropped while another stream still has to read what they hold: the memory must not be handed out before."""

import pytest
import torch

import ff_common as F
from paper_2002_09481_amd import binding as ax
from paper_2002_09481_amd import inputs as I
from paper_2002_09481_amd.feedforward import ExpertsFeedForward, FeedForward

pytestmark = pytest.mark.gpu

BUSY = 40_000_000  # cycles that the other stream is held: tens of milliseconds


def _dropped(make, use, s=None):
    """use(make(), stream) with what was made dropped at once; returns the results, after the current stream has filled whatever memory
    of those sizes it gets."""
    s = s or torch.cuda.Stream()
    held, shapes = make()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(BUSY)
    out = use(held, s)
    del held
    junk = [torch.full(sh, 7, dtype=d, device="cuda") for sh, d in shapes for _ in range(2)]
    torch.cuda.synchronize()
    assert all(bool((j == 7).all()) for j in junk)
    return out


def _tensors(b):
    w = [t for v in b.w.values() for t in ((v.codes, v.scales) if hasattr(v, "codes") else v)]
    return [(t.shape, t.dtype) for t in w]


@pytest.mark.parametrize("kind", [8, 4, "experts"])
def test_served_block_is_dropped(kind):
    g = F.gen(11)
    b = ExpertsFeedForward(256, 512, 4, 2, seed=1) if kind == "experts" else FeedForward(256, 1024, seed=1)
    x = F.randn(g, (40, 256), 1.0, torch.bfloat16).cuda()
    laid = lambda: b.quantized() if kind == "experts" else b.quantized(bits=kind)  # noqa: E731
    want = laid().forward(x)

    def make():
        q = laid()
        return q, _tensors(q)

    assert torch.equal(_dropped(make, lambda q, s: q.forward(x, stream=s)), want)


@pytest.mark.parametrize("experts", [False, True])
def test_trained_block_is_dropped(experts):
    g = F.gen(12)
    new = lambda: ExpertsFeedForward(256, 512, 4, 2, seed=2) if experts else FeedForward(256, 1024, seed=2)  # noqa: E731
    x, gy = (F.randn(g, (300, 256), 1.0, torch.bfloat16).cuda() for _ in range(2))
    b = new()
    want = b.forward(x, train=True), b.backward(gy)

    def make():
        b = new()
        return b, [(t.shape, t.dtype) for d in (b.params, b.grads, b.master) for t in d.values()]

    got = _dropped(make, lambda b, s: (b.forward(x, train=True, stream=s), b.backward(gy, stream=s)))
    assert all(torch.equal(a, c) for a, c in zip(got, want))


@pytest.mark.parametrize("kind", [8, 4, "experts"])
def test_block_is_dropped_after_its_weights_are_laid_out(kind):
    """The masters die with the block that they are laid out from; what is made on the other stream is used and dropped on this one."""
    g = F.gen(13)
    new = lambda: ExpertsFeedForward(256, 512, 4, 2, seed=3) if kind == "experts" else FeedForward(256, 1024, seed=3)  # noqa: E731
    laid = lambda b, s: b.quantized(stream=s) if kind == "experts" else b.quantized(stream=s, bits=kind)  # noqa: E731
    x = F.randn(g, (40, 256), 1.0, torch.bfloat16).cuda()
    want = laid(new(), None).forward(x)

    def make():
        b = new()
        return b, [(t.shape, t.dtype) for d in (b.params, b.master) for t in d.values()]

    s = torch.cuda.Stream()
    q = _dropped(make, laid, s)
    shapes = _tensors(q)
    torch.cuda._sleep(BUSY)
    y = q.forward(x)
    del q
    with torch.cuda.stream(s):
        junk = [torch.full(sh, 7, dtype=d, device="cuda") for sh, d in shapes for _ in range(2)]
    torch.cuda.synchronize()
    assert torch.equal(y, want) and all(bool((j == 7).all()) for j in junk)


@pytest.mark.parametrize("bits", [32, 8])
def test_optimizer_is_dropped(bits):
    """Parameters and states die with the optimizer, right after a step; the copies are what is looked at."""
    g = F.gen(14)
    p, gr = F.randn(g, (1 << 20,)).cuda(), F.randn(g, (1 << 20,)).cuda()
    copy = torch.zeros(1 << 20, dtype=torch.bfloat16, device="cuda")

    def make():
        opt = ax.AxAdamW([p.clone()], [gr], copies=[copy], bits=bits)
        return opt, [(t.shape, t.dtype) for t in opt.params + opt.m + opt.v + (opt.m_scales or []) + (opt.v_scales or [])]

    make()[0].step(1e-2, 1, weight_decay=0.1)
    want = copy.clone()
    copy.zero_()
    _dropped(make, lambda opt, s: opt.step(1e-2, 1, weight_decay=0.1, stream=s))
    assert torch.equal(copy, want)
    opt = make()[0]
    opt.step(1e-2, 1)
    want = [t.clone() for t in opt.states()[1]]

    def stepped():
        opt, shapes = make()
        opt.step(1e-2, 1)
        return opt, shapes

    if bits == 8:
        assert torch.equal(_dropped(stepped, lambda opt, s: opt.states(stream=s))[1][0], want[0])


def test_lookup_layer_is_dropped():
    layer = I.Layer("drop", 4, 28, 28, 64, 3, 3, 72, 1, 1, x_dist="relu", w_dist="normal")
    x, w, q = I.make_operands(layer, 15)
    lut, desc = I.lut_truncated(4), ax._conv_desc(x.shape, w.shape, 1, 1)
    xd = torch.from_numpy(x).cuda()

    def make():
        h = ax.AxLayer(desc, q)
        p = h.prepare(torch.from_numpy(w).cuda(), ax.lut_to_device(lut))
        return h, [(p.shape, p.dtype), (w.shape, torch.uint8), ((65536,), torch.int16)]

    want = make()[0].run(xd)
    got = _dropped(make, lambda h, s: h.run(xd, stream=s))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
