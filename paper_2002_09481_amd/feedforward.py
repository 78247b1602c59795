"""A pre-norm feed-forward block trained in float and served in 8 bits: the feed-forward operators of the library as they are
used together.

    t = x + residual          the residual stream (x itself without a residual)
    n = norm(t)               root-mean-square norm
    h = act(n wg) * (n wu)    gated projections
    y = h wd + bias + t       product back into the stream

Training keeps float32 master parameters and lets the optimizer's step write the copies that the products read, in the block's
type (bfloat16, or float32, where the masters are read themselves).  Serving takes 8-bit codes: the norm emits them with a
scale a row, weights are laid out once as [outputs, inputs] codes with a scale an output.
"""

from __future__ import annotations

import contextlib
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
            return ax._on_stream(self.forward, stream, x, residual, train)
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
            return ax._on_stream(self.backward, stream, gy)
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

    def quantized(self, stream=None):
        """The block in 8 bits, from the present parameters."""
        return QuantizedFeedForward(self, stream=stream)


class QuantizedFeedForward:
    """The block on int8 codes, forward only.  The residual stream keeps the block's type."""

    def __init__(self, block: FeedForward, stream=None):
        self.act, self.eps, self.dtype = block.act, block.eps, block.dtype
        with contextlib.nullcontext() if stream is None else torch.cuda.stream(stream):
            self.norm, self.bias = block.params["norm"].clone(), block.params["bias"].clone()
            self.w = {}
            for name in ("wg", "wu", "wd"):  # [inputs, outputs] -> codes [outputs, inputs], a scale an output
                codes, scales, _, _ = ax.ax_rmsnorm_q8(block.master[name].t().contiguous(), normalize=False)
                self.w[name] = (codes, scales)

    def forward(self, x, residual=None, stream=None):
        if stream is not None:
            return ax._on_stream(self.forward, stream, x, residual)
        codes, scales, t, _ = ax.ax_rmsnorm_q8(x, self.norm, residual=residual, eps=self.eps)
        t = x if t is None else t
        h = ax.ax_gated_q8(codes, scales, *self.w["wg"], *self.w["wu"], act=self.act, out_dtype=self.dtype)
        hc, hs, _, _ = ax.ax_rmsnorm_q8(h, normalize=False)
        return ax.ax_matmul_q8(hc, hs, *self.w["wd"], bias=self.bias, residual=t, out_dtype=self.dtype)
