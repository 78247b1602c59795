"""Pre-norm feed-forward blocks trained in float and served in 8 or 4 bits: the feed-forward operators of the library as they are
used together.

    t = x + residual          the residual stream (x itself without a residual)
    n = norm(t)               root-mean-square norm
    h = act(n wg) * (n wu)    gated projections
    y = h wd + bias + t       product back into the stream

Training keeps float32 master parameters and lets the optimizer's step write the copies that the products read, in the block's
type (bfloat16, or float32, where the masters are read themselves).  Serving takes 8-bit codes: the norm emits them with a
scale a row, weights are laid out once as [outputs, inputs] codes with a scale an output.  Or weights of 4 bits with a scale for
each group of an output's inputs, with the norm's values as they are: half the bytes of a block that serves single tokens.

The same block of experts (ExpertsFeedForward): a router chooses k of them for every token,

    l = n wr,  w = the weights of the k largest logits
    y = t + sum over the chosen e of w_e (act(n wg_e) * (n wu_e)) wd_e

with the rows of the choices grouped by expert between the router and the sum.
"""

from __future__ import annotations

import math

import torch

from . import binding as ax


class FeedForward:
    """width: features of the stream; hidden: features between the projections; dtype: torch.bfloat16 or torch.float32;
    bits: of the optimizer's states (32 or 8)."""

    NAMES = ("wg", "wu", "wd", "norm", "bias")

    def __init__(self, width, hidden, act="silu", dtype=torch.bfloat16, eps=1e-5, bits=32, device="cuda", seed=0):
        self.width, self.hidden, self.act, self.dtype, self.eps = int(width), int(hidden), act, dtype, float(eps)
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        rand = lambda r, c: torch.randn((r, c), generator=g, device=device) / math.sqrt(r)  # noqa: E731
        self.master = {"wg": rand(width, hidden), "wu": rand(width, hidden), "wd": rand(hidden, width),
                       "norm": torch.ones(width, device=device), "bias": torch.zeros(width, device=device)}
        low = dtype != torch.float32
        self.params = {n: t.to(dtype) if low else t for n, t in self.master.items()}
        self.grads = {n: torch.zeros_like(t if n in ("norm", "bias") else self.params[n]) for n, t in self.master.items()}
        # the weights' gradients have the products' type, those of the vectors are float32: a step for each list
        self._opts = [ax.AxAdamW([self.master[n] for n in names], [self.grads[n] for n in names], bits=bits,
                                 copies=[self.params[n] for n in names] if low else None)
                      for names in (self.NAMES[:3], self.NAMES[3:])]
        self.steps = 0
        self._kept = None

    def forward(self, x, residual=None, train=False, stream=None):
        """y [rows, width]; with train, what backward needs is kept until it is called, in the place of what an earlier pass
        left."""
        if stream is not None:
            return ax._on_stream(self.forward, stream, x, residual, train, held=(self.params,))
        p = self.params
        n, t, rstd = ax.ax_rmsnorm(x, p["norm"], residual=residual, eps=self.eps, rstd_out=None if train else False)
        t = x if t is None else t
        h, g, u = ax.ax_gated(n, p["wg"], p["wu"], act=self.act, save=train)
        y, _ = ax.ax_matmul(h, p["wd"], bias=p["bias"], residual=t)
        if train:
            self._kept = (n, t, rstd, h, g, u)
        return y

    def backward(self, gy, stream=None):
        """The gradient of x (and of the residual); those of the parameters are left in self.grads."""
        if stream is not None:
            return ax._on_stream(self.backward, stream, gy, held=(self.params, self.grads))
        if self._kept is None:
            raise RuntimeError("backward needs a forward pass with train=True first")
        n, t, rstd, h, g, u = kept = self._kept
        self._kept = None
        here = torch.cuda.current_stream(gy.device)
        for k in kept:  # (of the forward pass's stream; they die before this one has read them)
            k.record_stream(here)
        p, d = self.params, self.grads
        gh, _, _ = ax.ax_matmul_backward(gy, h, p["wd"], gw_out=d["wd"], gb_out=d["bias"])
        gn, _, _ = ax.ax_gated_backward(gh, n, p["wg"], p["wu"], g, u, act=self.act, gwg_out=d["wg"], gwu_out=d["wu"])
        gx, _ = ax.ax_rmsnorm_backward(gn, t, p["norm"], rstd, gsum=gy, gw_out=d["norm"])
        return gx

    def step(self, lr, weight_decay=0.0, grad_scale=None, stream=None, **betas):
        """One AdamW step with the gradients of the last backward pass; the vectors are not decayed."""
        self.steps += 1
        for opt, wd in zip(self._opts, (weight_decay, 0.0)):
            opt.step(lr, self.steps, weight_decay=wd, grad_scale=grad_scale, stream=stream, **betas)

    def quantized(self, stream=None, bits=8, group=128):
        """The block in 8 or 4 bits, from the present parameters."""
        return QuantizedFeedForward(self, stream=stream, bits=bits, group=group)


def _reading(block, stream, call):
    """call(), which reads the block's parameters, on `stream`."""
    return call() if stream is None else ax._on_stream(call, stream, held=(block.params, block.master))


class QuantizedFeedForward:
    """The block on int8 codes (bits = 8), or with weights of 4 bits (4: a scale for every `group` inputs); forward only.  The
    residual stream keeps the block's type."""

    def __init__(self, block: FeedForward, stream=None, bits=8, group=128):
        if bits not in (8, 4):
            raise ValueError("bits must be 8 or 4")
        self.act, self.eps, self.dtype, self.bits = block.act, block.eps, block.dtype, bits

        def lay_out():
            w = {}
            for name in ("wg", "wu", "wd"):  # [inputs, outputs] -> codes [outputs, inputs], a scale an output (or group)
                t = block.master[name].t().contiguous()
                w[name] = ax.ax_quantize_q4(t, group=group) if bits == 4 else ax.ax_rmsnorm_q8(t, normalize=False)[:2]
            return block.params["norm"].clone(), block.params["bias"].clone(), w

        self.norm, self.bias, self.w = _reading(block, stream, lay_out)

    def forward(self, x, residual=None, stream=None):
        if stream is not None:
            return ax._on_stream(self.forward, stream, x, residual, held=(self.norm, self.bias, self.w))
        if self.bits == 4:
            n, t, _ = ax.ax_rmsnorm(x, self.norm, residual=residual, eps=self.eps, rstd_out=False)
            h = ax.ax_gated_q4(n, self.w["wg"], self.w["wu"], act=self.act)
            return ax.ax_matmul_q4(h, self.w["wd"], bias=self.bias, residual=x if t is None else t)
        codes, scales, t, _ = ax.ax_rmsnorm_q8(x, self.norm, residual=residual, eps=self.eps)
        t = x if t is None else t
        h = ax.ax_gated_q8(codes, scales, *self.w["wg"], *self.w["wu"], act=self.act, out_dtype=self.dtype)
        hc, hs, _, _ = ax.ax_rmsnorm_q8(h, normalize=False)
        return ax.ax_matmul_q8(hc, hs, *self.w["wd"], bias=self.bias, residual=t, out_dtype=self.dtype)


class ExpertsFeedForward:
    """The block of experts.  width: features of the stream; hidden: features between an expert's projections; k: experts a token
    takes; normalize: whether their weights add up to one (the softmax over the chosen) or not (over all experts).  dtype, eps and
    bits as FeedForward.  Logits are float32."""

    NAMES = ("router", "wg", "wu", "wd", "norm")

    def __init__(self, width, hidden, experts, k, act="silu", dtype=torch.bfloat16, eps=1e-5, bits=32, normalize=True, device="cuda",
                 seed=0):
        self.width, self.hidden, self.experts, self.k, self.normalize = int(width), int(hidden), int(experts), int(k), bool(normalize)
        self.act, self.dtype, self.eps = act, dtype, float(eps)
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        rand = lambda *s: torch.randn(s, generator=g, device=device) / math.sqrt(s[-2])  # noqa: E731
        self.master = {"router": rand(width, experts), "wg": rand(experts, width, hidden), "wu": rand(experts, width, hidden),
                       "wd": rand(experts, hidden, width), "norm": torch.ones(width, device=device)}
        low = dtype != torch.float32
        self.params = {n: t.to(dtype) if low else t for n, t in self.master.items()}
        self.grads = {n: torch.zeros_like(t if n == "norm" else self.params[n]) for n, t in self.master.items()}
        self._opts = [ax.AxAdamW([self.master[n] for n in names], [self.grads[n] for n in names], bits=bits,
                                 copies=[self.params[n] for n in names] if low else None)
                      for names in (self.NAMES[:4], self.NAMES[4:])]
        self.steps = 0
        self._kept = None

    def forward(self, x, residual=None, train=False, stream=None):
        """y [tokens, width]; with train, what backward needs is kept until it is called, in the place of what an earlier pass
        left."""
        if stream is not None:
            return ax._on_stream(self.forward, stream, x, residual, train, held=(self.params,))
        p = self.params
        n, t, rstd = ax.ax_rmsnorm(x, p["norm"], residual=residual, eps=self.eps, rstd_out=None if train else False)
        t = x if t is None else t
        logits, _ = ax.ax_matmul(n, p["router"], out_dtype=torch.float32)
        experts, weights, offsets, rows, tokens = ax.ax_route(logits, self.k, normalize=self.normalize)
        h, g, u = ax.ax_gated_experts(n, p["wg"], p["wu"], offsets, tokens, act=self.act, save=train)
        d, _ = ax.ax_matmul_experts(h, p["wd"], offsets)
        y = ax.ax_combine(d, rows, weights, residual=t)
        if train:
            self._kept = (n, t, rstd, logits, experts, weights, offsets, rows, tokens, h, g, u, d)
        return y

    def backward(self, gy, stream=None):
        """The gradient of x (and of the residual); those of the parameters are left in self.grads."""
        if stream is not None:
            return ax._on_stream(self.backward, stream, gy, held=(self.params, self.grads))
        if self._kept is None:
            raise RuntimeError("backward needs a forward pass with train=True first")
        n, t, rstd, logits, experts, weights, offsets, rows, tokens, h, g, u, d = kept = self._kept
        self._kept = None
        here = torch.cuda.current_stream(gy.device)
        for k in kept:  # (of the forward pass's stream; they die before this one has read them)
            k.record_stream(here)
        p, out = self.params, self.grads
        gd, gweights = ax.ax_combine_backward(gy, d, rows, weights)
        gh, _ = ax.ax_matmul_experts_backward(gd, h, p["wd"], offsets, gw_out=out["wd"])
        grows, _, _ = ax.ax_gated_experts_backward(gh, n, p["wg"], p["wu"], g, u, offsets, tokens, act=self.act, gwg_out=out["wg"],
                                                   gwu_out=out["wu"])
        glogits = ax.ax_route_backward(gweights, logits, experts, weights, normalize=self.normalize)
        # (the router's product takes its gradient in its operands' type)
        gn, _, _ = ax.ax_matmul_backward(glogits.to(self.dtype), n, p["router"], gw_out=out["router"], gb_out=False)
        gn = ax.ax_combine(grows, rows, residual=gn, y_out=gn)
        gx, _ = ax.ax_rmsnorm_backward(gn, t, p["norm"], rstd, gsum=gy, gw_out=out["norm"])
        return gx

    def step(self, lr, weight_decay=0.0, grad_scale=None, stream=None, **betas):
        """One AdamW step with the gradients of the last backward pass; the norm is not decayed."""
        self.steps += 1
        for opt, wd in zip(self._opts, (weight_decay, 0.0)):
            opt.step(lr, self.steps, weight_decay=wd, grad_scale=grad_scale, stream=stream, **betas)

    def quantized(self, stream=None, group=128):
        """The block with experts in 4 bits, from the present parameters."""
        return QuantizedExperts(self, stream=stream, group=group)


class QuantizedExperts:
    """The block of experts with their weights in 4 bits, a scale for every `group` inputs; forward only.  The router keeps the
    block's type."""

    def __init__(self, block: ExpertsFeedForward, stream=None, group=128):
        self.act, self.eps, self.dtype, self.k, self.normalize = block.act, block.eps, block.dtype, block.k, block.normalize

        def lay_out():
            w = {name: ax.ax_quantize_q4(block.master[name].transpose(1, 2).contiguous(), group=group) for name in ("wg", "wu", "wd")}
            return block.params["norm"].clone(), block.params["router"].clone(), w

        self.norm, self.router, self.w = _reading(block, stream, lay_out)

    def forward(self, x, residual=None, stream=None):
        if stream is not None:
            return ax._on_stream(self.forward, stream, x, residual, held=(self.norm, self.router, self.w))
        n, t, _ = ax.ax_rmsnorm(x, self.norm, residual=residual, eps=self.eps, rstd_out=False)
        logits, _ = ax.ax_matmul(n, self.router, out_dtype=torch.float32)
        _, weights, offsets, rows, tokens = ax.ax_route(logits, self.k, normalize=self.normalize)
        h = ax.ax_gated_q4(n, self.w["wg"], self.w["wu"], act=self.act, offsets=offsets, tokens=tokens)
        d = ax.ax_matmul_q4(h, self.w["wd"], offsets=offsets)
        return ax.ax_combine(d, rows, weights, residual=x if t is None else t)
