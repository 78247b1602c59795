"""Calls on a stream that is not the current one, while the current stream still has work with memory that was freed: the calls
wait for nothing, so what they allocate must not be that memory."""

import pytest
import torch

import ff_common as F
from paper_2002_09481_amd import binding as ax
from paper_2002_09481_amd import inputs as I
from paper_2002_09481_amd.feedforward import FeedForward

pytestmark = pytest.mark.gpu

BUSY = 40_000_000  # cycles that the current stream is held: tens of milliseconds


def _while_the_current_stream_reads(shapes_dtypes, call):
    """call() while the current stream waits with a read of freed blocks of these shapes; returns what it read."""
    torch.cuda.synchronize()
    freed = [torch.full(s, 3, dtype=d, device="cuda") for s, d in shapes_dtypes]
    read = [torch.empty_like(t) for t in freed]
    torch.cuda.synchronize()
    torch.cuda._sleep(BUSY)
    for r, t in zip(read, freed):
        r.copy_(t)
    del t, freed
    out = call()
    torch.cuda.synchronize()
    assert all(bool((r == 3).all()) for r in read)
    return out


def test_products_on_another_stream_leave_freed_memory_alone():
    g, M, K, N = F.gen(2), 512, 1000, 1024
    x, w, wu = (F.randn(g, s).cuda() for s in ((M, K), (K, N), (K, N)))
    gy = F.randn(g, (M, N)).cuda()
    want = ax.ax_gated(x, w, wu, save=True)
    grads = ax.ax_gated_backward(gy, x, w, wu, want[1], want[2])
    s = torch.cuda.Stream()
    outs = [((M, N), torch.float32)] * 4 + [((M, K), torch.float32), ((K, N), torch.float32), ((K, N), torch.float32)]
    spare = [((1 << 22,), torch.uint8), ((1 << 24,), torch.uint8), ((1 << 25,), torch.uint8)]  # (workspaces)

    def call():
        h, g_, u = ax.ax_gated(x, w, wu, save=True, stream=s)
        return (h, g_, u), ax.ax_gated_backward(gy, x, w, wu, g_, u, stream=s)

    got, back = _while_the_current_stream_reads(outs + spare, call)
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and all(torch.equal(a, b) for a, b in zip(back, grads))


def test_norm_and_states_on_another_stream_leave_freed_memory_alone():
    g, rows, cols = F.gen(3), 2000, 1000
    x, w = F.randn(g, (rows, cols)).cuda(), torch.ones(cols, device="cuda")
    opt = ax.AxAdamW([x.clone()], [x.clone()], bits=8)
    opt.step(1e-3, 1)
    want = ax.ax_rmsnorm(x, w, residual=x), ax.ax_rmsnorm_q8(x, w, values=True), opt.states()
    s = torch.cuda.Stream()
    outs = [((rows, cols), torch.float32)] * 5 + [((rows, cols), torch.int8), ((rows,), torch.float32), ((rows,), torch.float32)]
    got = _while_the_current_stream_reads(outs, lambda: (ax.ax_rmsnorm(x, w, residual=x, stream=s),
                                                         ax.ax_rmsnorm_q8(x, w, values=True, stream=s), opt.states(stream=s)))
    for a, b in zip(got, want):
        for u, v in zip(a, b):
            assert (u is None and v is None) or (torch.equal(u, v) if isinstance(u, torch.Tensor) else torch.equal(u[0], v[0]))


def test_what_a_call_on_another_stream_took_may_be_dropped():
    """The operands die right after the call: their memory must not be handed out while the other stream still has to read it."""
    g, M, K, N = F.gen(4), 256, 512, 512
    x, w = F.randn(g, (M, K)).cuda(), F.randn(g, (K, N), 0.05).cuda()
    want, _ = ax.ax_matmul(x, w)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    a, b = x.clone(), w.clone()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(BUSY)
    y, _ = ax.ax_matmul(a, b, stream=s)
    del a, b
    junk = [torch.full((M, K), 7.0, device="cuda"), torch.full((K, N), 7.0, device="cuda")]
    s.synchronize()
    assert torch.equal(y, want) and bool((junk[0] == 7).all())


def test_lookup_layers_on_another_stream_leave_freed_memory_alone():
    x, w, q = I.make_operands(I.Layer("side", 4, 28, 28, 64, 3, 3, 72, 1, 1, x_dist="relu", w_dist="normal"), 1)
    lut = ax.lut_to_device(I.lut_truncated(4))
    xd, wd = torch.from_numpy(x).cuda(), torch.from_numpy(w).cuda()
    acc, y = ax.ax_conv2d(xd, wd, lut, 1, 1, q)
    gx, gw = ax.ax_conv2d_backward(xd, wd, y, 1, 1, q)
    s = torch.cuda.Stream()
    need = ax.ax_conv2d_workspace_bytes(x.shape, w.shape, 1, 1)
    outs = [(acc.shape, torch.int32), (y.shape, torch.float32), ((need,), torch.uint8), (gx.shape, torch.float32), (gw.shape, torch.float32),
            ((1 << 24,), torch.uint8)]
    got = _while_the_current_stream_reads(outs, lambda: ax.ax_conv2d(xd, wd, lut, 1, 1, q, stream=s) +
                                          ax.ax_conv2d_backward(xd, wd, y, 1, 1, q, stream=s))
    assert torch.equal(got[0], acc) and torch.equal(got[1], y)
    assert torch.equal(got[2], gx) and torch.equal(got[3], gw)


def test_backward_pass_on_another_stream_than_the_forward():
    """The forward pass's results die as soon as the backward pass is enqueued; the current stream's next tensors must not take
    their place."""
    b, g = FeedForward(256, 1024, dtype=torch.bfloat16, seed=3), F.gen(5)
    x, gy = (F.randn(g, (300, 256), 1.0, torch.bfloat16).cuda() for _ in range(2))
    b.forward(x, train=True)
    want = [b.backward(gy).clone()] + [b.grads[k].clone() for k in b.NAMES]
    for t in b.grads.values():
        t.zero_()
    b.forward(x, train=True)
    shapes = [(t.shape, t.dtype) for t in b._kept]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(BUSY)
    gx = b.backward(gy, stream=s)
    junk = [torch.full(sh, 9, dtype=d, device="cuda") for sh, d in shapes for _ in range(2)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, c) for a, c in zip([gx] + [b.grads[k] for k in b.NAMES], want))
    assert all(bool((j == 9).all()) for j in junk)
