"""The feed-forward block that runs the operators together: a training step against 64-bit autograd, serving in 8 bits, other
streams, capture into a graph."""

import pytest
import torch

import ff_common as F
from paper_2002_09481_amd.feedforward import FeedForward

pytestmark = pytest.mark.gpu


def _block(dtype, **kw):
    b = FeedForward(96, 264, dtype=dtype, seed=3, **kw)
    b.params["norm"].mul_(1.25)
    if dtype != torch.float32:
        b.master["norm"].copy_(b.params["norm"])
    return b


def _plain(b, x, r):
    p = {k: v.detach().cpu().double().requires_grad_() for k, v in b.params.items()}
    x, r = x.cpu().double().requires_grad_(), r.cpu().double().requires_grad_()
    t = x + r
    n = t / torch.sqrt((t ** 2).mean(dim=1, keepdim=True) + b.eps) * p["norm"]
    h = torch.nn.functional.silu(n @ p["wg"]) * (n @ p["wu"])
    return h @ p["wd"] + p["bias"] + t, p, x, r


@pytest.mark.parametrize("dt,bits", [("f32", 32), ("bf16", 32), ("bf16", 8)])
def test_training_step(dt, bits):
    dtype = F.DT[dt]
    b = _block(dtype, bits=bits)
    g = F.gen(1)
    x, r, gy = (F.randn(g, (37, 96), 1.0, dtype).cuda() for _ in range(3))
    y = b.forward(x, r, train=True)
    want, p, xd, rd = _plain(b, x, r)
    want.backward(gy.cpu().double())
    # relative, in the 2-norm: five float32 stages, or eight roundings to bf16 (2^-8 each at most, in and out of the products)
    tol = 8 * 2.0 ** -8 if dt == "bf16" else 300 * F.U
    near = lambda a, e: float((a.cpu().double() - e).norm() / e.norm())  # noqa: E731
    assert near(y, want.detach()) <= tol
    before = {k: v.clone() for k, v in b.master.items()}
    gx = b.backward(gy)
    assert near(gx, xd.grad) <= tol and torch.equal(xd.grad, rd.grad)
    for k in b.NAMES:
        assert near(b.grads[k], p[k].grad) <= tol, k
    b.step(1e-3, weight_decay=0.1)
    for k in b.NAMES:  # the first step moves every parameter by lr against its gradient's sign
        move = b.master[k] - before[k] * (1 - 1e-3 * (0.1 if k.startswith("w") else 0))
        assert float((move + 1e-3 * torch.sign(b.grads[k].float())).abs().max()) <= 2e-6 + 1e-3 * 1e-8 / float(b.grads[k].float().abs().min().clamp(min=1e-30)), k
        assert torch.equal(b.params[k], b.master[k].to(dtype))
    with pytest.raises(RuntimeError):
        b.backward(gy)


def test_training_lowers_the_loss():
    b = _block(torch.bfloat16, bits=8)
    g = F.gen(2)
    x, want = F.randn(g, (256, 96), 1.0, torch.bfloat16).cuda(), F.randn(g, (256, 96), 1.0, torch.bfloat16).cuda()
    losses = []
    for _ in range(30):
        e = b.forward(x, train=True).float() - want.float()
        losses.append(float(e.square().mean()))
        b.backward((e * (2 / e.numel())).to(torch.bfloat16))
        b.step(3e-3)
    assert losses[-1] < 0.6 * losses[0] and all(v == v for v in losses)


@pytest.mark.parametrize("rows", [1, 5, 70])
def test_serving_in_8_bits(rows):
    b = _block(torch.bfloat16)
    g = F.gen(4)
    x, r = (F.randn(g, (rows, 96), 1.0, torch.bfloat16).cuda() for _ in range(2))
    q = b.quantized()
    y, want = q.forward(x, r), _plain(b, x, r)[0].detach()
    # codes of 127 levels: at most 1 / 254 of a row's largest value each, for the activations twice and the weights
    t = (x.cpu().double() + r.cpu().double())
    assert float((y.cpu().double() - want).norm() / (want - t).norm()) <= 4 * 4.5 / 254
    assert torch.equal(y[:1], q.forward(x[:1].contiguous(), r[:1].contiguous()))  # a token does not depend on its batch


def test_another_stream_and_a_graph():
    b = _block(torch.bfloat16)
    q = b.quantized()
    g = F.gen(5)
    x, r, gy = (F.randn(g, (40, 96), 1.0, torch.bfloat16).cuda() for _ in range(3))
    want = [q.forward(x, r), b.forward(x, r, train=True)]
    want.append(b.backward(gy))
    want += [b.grads[k].clone() for k in b.NAMES]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = [q.forward(x, r), b.forward(x, r, train=True)]
        got.append(b.backward(gy))
    s.synchronize()
    got += [b.grads[k].clone() for k in b.NAMES]
    assert all(torch.equal(a, c) for a, c in zip(got, want))

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = [q.forward(x, r), b.forward(x, r, train=True)]
        out.append(b.backward(gy))
    for k in range(4):
        for t in out:
            t.zero_()
        for t in b.grads.values():
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        eager = q.forward(x, r)  # the program's own work between replays
        torch.cuda.synchronize()
        assert torch.equal(eager, want[0])
        assert all(torch.equal(a, c) for a, c in zip(out + [b.grads[n] for n in b.NAMES], want))
