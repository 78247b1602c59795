"""The block of experts that runs its operators together, and the blocks served with weights of 4 bits: a training step against 64-bit
autograd, serving, other streams, capture into a graph."""

import pytest
import torch

import ff_common as F
from paper_2002_09481_amd import binding as ax
from paper_2002_09481_amd.feedforward import ExpertsFeedForward, FeedForward

pytestmark = pytest.mark.gpu


def _block(dtype, **kw):
    b = ExpertsFeedForward(96, 136, 6, 2, dtype=dtype, seed=3, **kw)
    b.params["norm"].mul_(1.25)
    if dtype != torch.float32:
        b.master["norm"].copy_(b.params["norm"])
    return b


def _choices(b, x, r):
    """The experts that the block's own router takes (a tie of rounded logits is not for the plain form to decide)."""
    n, _, _ = ax.ax_rmsnorm(x, b.params["norm"], residual=r, eps=b.eps)
    logits, _ = ax.ax_matmul(n, b.params["router"], out_dtype=torch.float32)
    return ax.ax_route(logits, b.k)[0].cpu().long()


def _plain(b, x, r, experts, weights=None):
    p = {k: v.detach().cpu().double().requires_grad_() for k, v in (weights or b.params).items()}
    x, r = x.cpu().double().requires_grad_(), r.cpu().double().requires_grad_()
    t = x + r
    n = t / torch.sqrt((t ** 2).mean(dim=1, keepdim=True) + b.eps) * p["norm"]
    logits = n @ p["router"]
    w = torch.softmax(torch.gather(logits, 1, experts), dim=1) if b.normalize else torch.gather(torch.softmax(logits, dim=1), 1, experts)
    y = t
    for j in range(b.k):
        e = experts[:, j]
        h = torch.nn.functional.silu(torch.einsum("tc,tch->th", n, p["wg"][e])) * torch.einsum("tc,tch->th", n, p["wu"][e])
        y = y + w[:, j:j + 1] * torch.einsum("th,thc->tc", h, p["wd"][e])
    return y, t, p, x, r


near = lambda a, e: float((a.cpu().double() - e).norm() / e.norm())  # noqa: E731


@pytest.mark.parametrize("normalize", [True, False])
@pytest.mark.parametrize("tokens", [1, 9, 300])
@pytest.mark.parametrize("dt,bits", [("f32", 32), ("bf16", 32), ("bf16", 8)])
def test_training_step(dt, bits, tokens, normalize):
    dtype = F.DT[dt]
    b = _block(dtype, bits=bits, normalize=normalize)
    g = F.gen(tokens)
    x, r, gy = (F.randn(g, (tokens, 96), 1.0, dtype).cuda() for _ in range(3))
    y = b.forward(x, r, train=True)
    want, t, p, xd, rd = _plain(b, x, r, _choices(b, x, r))
    want.backward(gy.cpu().double())
    # relative, in the 2-norm: seven float32 stages, or eleven roundings to bf16 (2^-8 each at most, in and out of the products)
    tol = 11 * 2.0 ** -8 if dt == "bf16" else 500 * F.U
    assert near(y, want.detach()) <= tol
    before = {k: v.clone() for k, v in b.master.items()}
    gx = b.backward(gy)
    assert near(gx, xd.grad) <= tol and torch.equal(xd.grad, rd.grad)
    for k in b.NAMES:
        assert near(b.grads[k], p[k].grad) <= tol, k
    b.step(1e-3, weight_decay=0.1)
    for k in b.NAMES:
        assert bool((b.master[k] != before[k]).any()) and torch.equal(b.params[k], b.master[k].to(dtype))
    with pytest.raises(RuntimeError):
        b.backward(gy)


@pytest.mark.parametrize("tokens", [1, 5, 400])
def test_serving_in_4_bits(tokens):
    b, dense = _block(torch.bfloat16), FeedForward(96, 264, seed=4)
    g = F.gen(tokens)
    x, r = (F.randn(g, (tokens, 96), 1.0, torch.bfloat16).cuda() for _ in range(2))
    q = b.quantized(group=32)
    # the same block from the values that the codes stand for: what is left are roundings to bf16, eleven of them at most
    values = dict(b.params, **{k: w.values().transpose(1, 2) for k, w in q.w.items()})
    want, t, *_ = _plain(b, x, r, _choices(b, x, r), weights=values)
    y = q.forward(x, r)
    assert y.shape == x.shape and near(y, want.detach()) <= 11 * 2.0 ** -8
    # codes of 4 bits: off by half a step of 1 / 7 of a group's largest at most
    for k, w in q.w.items():
        top = b.master[k].transpose(1, 2).abs().amax()
        assert float((values[k] - b.master[k]).abs().amax()) <= float(top) / 14 * 1.02
    s = dense.quantized(bits=4, group=64)
    v = {k: w.values().t().cpu().double() for k, w in s.w.items()}
    t = x.cpu().double() + r.cpu().double()
    n = t / torch.sqrt((t ** 2).mean(dim=1, keepdim=True) + dense.eps)
    want = t + (torch.nn.functional.silu(n @ v["wg"]) * (n @ v["wu"])) @ v["wd"]
    assert near(s.forward(x, r), want) <= 8 * 2.0 ** -8


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_a_batch_of_sequences(dt):
    """[batch, length, width] gives the bits of its rows."""
    b, g = _block(F.DT[dt]), F.gen(5)
    x, gy = (F.randn(g, (3, 7, 96), 1.0, F.DT[dt]).cuda() for _ in range(2))
    y, flat = b.forward(x, train=True), lambda t: t.view(21, -1)  # noqa: E731
    gx, grads = b.backward(gy), {k: v.clone() for k, v in b.grads.items()}
    assert y.shape == gx.shape == x.shape
    assert torch.equal(flat(y), b.forward(flat(x), train=True)) and torch.equal(flat(gx), b.backward(flat(gy)))
    assert all(torch.equal(v, b.grads[k]) for k, v in grads.items())
    q = b.quantized(group=64)
    assert torch.equal(flat(q.forward(x)), q.forward(flat(x)))


def test_two_calls_at_once():
    """One block's weights, two streams, other tokens and other choices on each."""
    b, g = _block(torch.bfloat16), F.gen(6)
    q = b.quantized(group=32)
    xs = [F.randn(g, (n, 96), 1.0, torch.bfloat16).cuda() for n in (700, 333)]
    want = [(b.forward(x), q.forward(x)) for x in xs]
    streams = [torch.cuda.Stream() for _ in xs]
    torch.cuda.synchronize()
    out = [[(b.forward(x, stream=s), q.forward(x, stream=s)) for x, s in zip(xs, streams)] for _ in range(5)]
    torch.cuda.synchronize()
    for both in out:
        for got, w in zip(both, want):
            assert all(torch.equal(a, e) for a, e in zip(got, w))


def test_refused_bits():
    with pytest.raises(ValueError):
        FeedForward(32, 32).quantized(bits=5)


@pytest.mark.parametrize("tokens", [3, 200])
def test_another_stream_and_a_graph(tokens):
    b = _block(torch.bfloat16)
    q = b.quantized()
    g = F.gen(5)
    x, r, gy = (F.randn(g, (tokens, 96), 1.0, torch.bfloat16).cuda() for _ in range(3))
    want = [q.forward(x, r), b.forward(x, r, train=True)]
    want.append(b.backward(gy))
    want += [b.grads[k].clone() for k in b.NAMES]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for way in ("argument", "current"):
        if way == "argument":
            got = [q.forward(x, r, stream=s), b.forward(x, r, train=True, stream=s), None]
            got[2] = b.backward(gy, stream=s)
        else:
            with torch.cuda.stream(s):
                got = [q.forward(x, r), b.forward(x, r, train=True)]
                got.append(b.backward(gy))
        s.synchronize()
        got += [b.grads[k].clone() for k in b.NAMES]
        assert all(torch.equal(a, c) for a, c in zip(got, want))
    assert torch.equal(b.quantized(stream=s).forward(x, r, stream=s), want[0])

    graph, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = [q.forward(x, r), b.forward(x, r, train=True)]
        out.append(b.backward(gy))
    with torch.cuda.graph(other):  # a second one, replayed between the replays of the first
        out2 = [q.forward(r, x), b.forward(r, x, train=True)]
    want2 = [q.forward(r, x), b.forward(r, x)]
    for k in range(4):
        for t in out + out2:
            t.zero_()
        for t in b.grads.values():
            t.zero_()
        graph.replay()
        other.replay()
        torch.cuda.synchronize()
        eager = q.forward(x, r)  # the program's own work between replays
        torch.cuda.synchronize()
        assert torch.equal(eager, want[0])
        assert all(torch.equal(a, c) for a, c in zip(out + [b.grads[n] for n in b.NAMES], want))
        assert all(torch.equal(a, c) for a, c in zip(out2, want2))


def test_a_graph_of_another_choice():
    """A captured block follows the router: other tokens, other sizes of the experts, the same graph."""
    b = _block(torch.float32)
    g = F.gen(8)
    x = F.randn(g, (50, 96)).cuda()
    b.forward(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = b.forward(x)
    for k in range(4):
        x.copy_(F.randn(g, (50, 96)).cuda() + (3.0 * b.params["router"][:, k] if k else 0.0))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, b.forward(x))
