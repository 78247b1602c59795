"""Performance cases of the operators around a network's feed-forward blocks: the norm in front of a
block, the matrix products in it and the optimizer's step over its weights.

Every case is a dict of plain values; "op" names the operator and "way" the direction:

  norm    root-mean-square norm of rows, with the residual's addition in front
            forward    values out (what training and a float network take), with the sum and 1 / rms
            q8         8-bit codes with a scale a row out (what an 8-bit product takes)
            rows_q8    the same codes without the norm (hidden activations between two 8-bit products)
            backward   gradients of the rows and of the weight
  matmul  product with bias, activation and residual in the epilogue
            serve      the output alone
            train      the output and the value before the activation, kept for the backward pass
            backward   gradients of the input, the weight and the bias
  gated   gated feed-forward: act(x wg) * (x wu) in one pass
            serve / train / backward as above; train keeps both projections
  adamw   one step over all tensors of a few blocks, states in 32 or 8 bits

"dtype" is the operands' type: "f32", "bf16", or "q8" for 8-bit codes with scales (forward only, float
results in bf16).  Where `own` is false the operators are computed in their plain form, elementary torch
operations in 32 bits; where it is true, by this library's entry points.
"""

import math

import torch

own = False

DEV = "cuda" if torch.cuda.is_available() else "cpu"
EPS = 1e-5
BLOCK = 256  # elements that share a scale of an 8-bit optimizer state
ADAM = dict(lr=3e-4, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1, step=20)

MOST_FLOPS = 2.0 * 8192 * 4096 * 2 * 16384  # of one case
MOST_ELEMS = 8192 * 8192  # rows * columns of a norm


def listed():
    return [
        # one token of one sequence being decoded in 8 bits: nothing but latency
        dict(name="norm_token_q8", op="norm", way="q8", rows=1, cols=2048, dtype="bf16", residual=True),
        # a long prompt in front of an 8-bit block: bandwidth
        dict(name="norm_prompt_q8", op="norm", way="q8", rows=8192, cols=4096, dtype="bf16", residual=True),
        # a float32 network of 1000 features trained on an odd number of rows
        dict(name="norm_backward_odd", op="norm", way="backward", rows=6007, cols=1000, dtype="f32", residual=True),
        # a projection for one token: every weight is read once, for one row
        dict(name="matmul_token", op="matmul", way="serve", M=1, K=4096, N=4096, dtype="bf16", act="none", bias=True,
             residual=True, transposed=False),
        # an 8-bit projection back to the residual stream for a batch of ragged prompts
        dict(name="matmul_q8_ragged", op="matmul", way="serve", M=333, K=8192, N=2048, dtype="q8", act="none", bias=False,
             residual=True, transposed=True),
        # an ordinary layer of a training step, its activation fused
        dict(name="matmul_train", op="matmul", way="train", M=8192, K=2048, N=8192, dtype="bf16", act="gelu", bias=True,
             residual=False, transposed=False),
        # gradients of the 2048 -> 1000 classifier in float32, odd batch
        dict(name="matmul_backward_f32", op="matmul", way="backward", M=1531, K=2048, N=1000, dtype="f32", act="relu",
             bias=True, residual=False, transposed=False),
        # a few sequences decoded together in 8 bits
        dict(name="gated_batch_q8", op="gated", way="serve", M=17, K=4096, F=10240, dtype="q8", act="silu"),
        # the largest training step
        dict(name="gated_train", op="gated", way="train", M=8192, K=4096, F=16384, dtype="bf16", act="silu"),
        # its gradients, for a smaller block and an odd number of tokens
        dict(name="gated_backward", op="gated", way="backward", M=4101, K=2048, F=5512, dtype="bf16", act="silu"),
        # a toy network's weights: many small tensors, latency
        dict(name="adamw_small", op="adamw", blocks=3, width=256, ff=1000, dtype="f32", bits=32),
        # float32 master weights of large blocks with 16-bit gradients and copies, states in 8 bits
        dict(name="adamw_large_8bit", op="adamw", blocks=2, width=4096, ff=12288, dtype="mixed", bits=8),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm; every other one is made odd."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    n = max(lo, min(hi, n | 1 if rng.random() < 0.5 else -(-n // 8) * 8))
    return n + 8 if n == 3072 else n


def draw(rng):
    op = rng.choice(["norm", "matmul", "gated", "adamw"])
    if op == "norm":
        way = rng.choice(["forward", "q8", "rows_q8", "backward"])
        cols = _log(rng, 64, 16384)
        c = dict(op=op, way=way, rows=_log(rng, 1, max(1, min(16384, MOST_ELEMS // cols))), cols=cols,
                 dtype=rng.choice(["bf16", "f32"]), residual=rng.random() < 0.5)
        if way == "rows_q8":
            c["residual"] = False
        return c
    if op == "matmul":
        way = rng.choice(["serve", "train", "backward"])
        dtype = rng.choice(["bf16", "f32", "q8"]) if way == "serve" else rng.choice(["bf16", "f32"])
        K, N = _log(rng, 64, 8192), _log(rng, 64, 8192)
        return dict(op=op, way=way, M=_log(rng, 1, 64) if way == "serve" and rng.random() < 0.5 else _log(rng, 1, 8192), K=K,
                    N=N, dtype=dtype, act=rng.choice(["none", "relu", "silu", "gelu"]), bias=rng.random() < 0.5,
                    residual=rng.random() < 0.5 and way != "backward", transposed=dtype == "q8" or rng.random() < 0.5)
    if op == "gated":
        way = rng.choice(["serve", "train", "backward"])
        dtype = rng.choice(["bf16", "f32", "q8"]) if way == "serve" else rng.choice(["bf16", "f32"])
        K = _log(rng, 64, 4096)
        return dict(op=op, way=way, M=_log(rng, 1, 64) if way == "serve" and rng.random() < 0.5 else _log(rng, 1, 4096), K=K,
                    F=_log(rng, 64, 12288), dtype=dtype, act=rng.choice(["relu", "silu", "gelu"]))
    return dict(op=op, blocks=rng.randint(1, 3), width=_log(rng, 64, 2048), ff=_log(rng, 64, 8192),
                dtype=rng.choice(["f32", "mixed", "bf16"]), bits=rng.choice([8, 32]))


# ---- inputs, made from the seed ---------------------------------------------------------------


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 7919 + 13)
    return g


def _type(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _randn(g, shape, scale, dtype):
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)


def _codes(g, rows, cols):
    """8-bit codes of normal rows, and a scale a row."""
    t = torch.randn((rows, cols), generator=g, device=DEV)
    amax = t.abs().amax(dim=1, keepdim=True)
    return torch.round(t * (127.0 / amax)).to(torch.int8), (amax / 127.0).reshape(-1)


def _tensor_shapes(c):
    """The tensors of `blocks` feed-forward blocks: norm weight, both projections, product back, its bias."""
    d, f = c["width"], c["ff"]
    return [(d,), (d, f), (d, f), (f, d), (d,)] * c["blocks"]


def prepare(case, seed):
    c, g = case, _gen(seed)
    s = {"case": c}
    if c["op"] == "norm":
        dt, shape = _type(c["dtype"]), (c["rows"], c["cols"])
        x = torch.randn(shape, generator=g, device=DEV)
        x[:, :: max(1, c["cols"] // 8)] *= 12.0  # a few channels that stand out
        s["x"] = x.to(dt)
        s["w"] = (1.0 + 0.1 * torch.randn((c["cols"],), generator=g, device=DEV)).to(dt)
        s["r"] = _randn(g, shape, 1.0, dt) if c["residual"] else None
        if c["way"] == "backward":
            s["rstd"] = torch.rsqrt(s["x"].float().square().mean(dim=1) + EPS)
            s["gy"] = _randn(g, shape, 0.02, dt)
    elif c["op"] == "matmul":
        M, K, N, dt = c["M"], c["K"], c["N"], _type(c["dtype"])
        if c["dtype"] == "q8":
            s["x"], s["xs"] = _codes(g, M, K)
            s["w"], ws = _codes(g, N, K)
            s["ws"] = ws / math.sqrt(K)
        else:
            s["x"] = _randn(g, (M, K), 1.0, dt)
            s["w"] = _randn(g, (N, K) if c["transposed"] else (K, N), 1.0 / math.sqrt(K), dt)
        s["b"] = _randn(g, (N,), 0.5, dt) if c["bias"] else None
        s["r"] = _randn(g, (M, N), 1.0, dt) if c["residual"] else None
        if c["way"] == "backward":
            s["gy"] = _randn(g, (M, N), 0.02, dt)
            s["z"] = _randn(g, (M, N), 1.0, dt) if c["act"] != "none" else None
    elif c["op"] == "gated":
        M, K, F, dt = c["M"], c["K"], c["F"], _type(c["dtype"])
        if c["dtype"] == "q8":
            s["x"], s["xs"] = _codes(g, M, K)
            for n in ("wg", "wu"):
                s[n], ws = _codes(g, F, K)
                s[n + "s"] = ws / math.sqrt(K)
        else:
            s["x"] = _randn(g, (M, K), 1.0, dt)
            s["wg"], s["wu"] = (_randn(g, (K, F), 1.0 / math.sqrt(K), dt) for _ in range(2))
        if c["way"] == "backward":
            s["gh"], s["g"], s["u"] = _randn(g, (M, F), 0.02, dt), _randn(g, (M, F), 1.0, dt), _randn(g, (M, F), 1.0, dt)
    else:
        pt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
        gt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
        shapes = _tensor_shapes(c)
        s["p"] = [_randn(g, sh, 0.02, pt) for sh in shapes]
        s["g"] = [_randn(g, sh, 1e-3, gt) for sh in shapes]
        s["m"] = [_randn(g, sh, 3e-4, torch.float32) for sh in shapes]
        s["v"] = [torch.randn(sh, generator=g, device=DEV).square_().mul_(1e-6) for sh in shapes]
        s["copy"] = [t.to(torch.bfloat16) for t in s["p"]] if c["dtype"] == "mixed" else None
        if c["bits"] == 8:
            s["m"], s["ms"] = zip(*[_encode_m(t) for t in s["m"]])
            s["v"], s["vs"] = zip(*[_encode_v(t) for t in s["v"]])
        if own:  # the optimizer object that a program keeps from step to step
            from paper_2002_09481_amd import binding as ax

            s["opt"] = ax.AxAdamW(s["p"], s["g"], s["m"], s["v"], s.get("ms"), s.get("vs"), copies=s["copy"])
    return s


# ---- plain forms --------------------------------------------------------------------------------


def _act(z, act):
    if act == "relu":
        return z.clamp(min=0.0)
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return z


def _act_grad(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "silu":
        sg = 1.0 / (1.0 + torch.exp(-z))
        return sg * (1.0 + z * (1.0 - sg))
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    return torch.ones_like(z)


def _encode_m(m):
    """First moments in 8 bits: m = scale * c |c| / 127^2, a scale for every BLOCK elements, its largest |m|."""
    n = m.numel()
    b = torch.nn.functional.pad(m.reshape(-1), (0, -n % BLOCK)).view(-1, BLOCK)
    scale = b.abs().amax(dim=1)
    inv = torch.where(scale >= 2.0 ** -126, torch.ones_like(scale) / scale, torch.zeros_like(scale))
    code = torch.round(torch.sqrt(b.abs() * inv[:, None]) * 127.0)
    code = torch.where(b < 0, -code, code)
    return code.to(torch.int8).reshape(-1)[:n].view(m.shape), scale


def _decode_m(code, scale):
    n = code.numel()
    r = torch.nn.functional.pad(code.reshape(-1), (0, -n % BLOCK)).view(-1, BLOCK).float() * (1.0 / 127.0)
    return (r * r.abs() * scale[:, None]).reshape(-1)[:n].view(code.shape)


def _encode_v(v):
    """Second moments in 8 bits: v = scale * (c / 255)^4; a value above zero never gets code zero."""
    n = v.numel()
    b = torch.nn.functional.pad(v.reshape(-1), (0, -n % BLOCK)).view(-1, BLOCK)
    scale = b.amax(dim=1)
    inv = torch.where(scale >= 2.0 ** -126, torch.ones_like(scale) / scale, torch.zeros_like(scale))
    code = torch.round(torch.sqrt(torch.sqrt(b * inv[:, None])) * 255.0)
    code = torch.where((b > 0) & (inv[:, None] > 0), code.clamp(min=1.0), code)
    return code.to(torch.uint8).reshape(-1)[:n].view(v.shape), scale


def _decode_v(code, scale):
    n = code.numel()
    r = torch.nn.functional.pad(code.reshape(-1), (0, -n % BLOCK)).view(-1, BLOCK).float() * (1.0 / 255.0)
    r = r * r
    return (r * r * scale[:, None]).reshape(-1)[:n].view(code.shape)


def _adam_update(p, g, m, v, F):
    """One tensor's step in the type of p, g, m and v; F: factors of the step."""
    m = F["b1"] * m + F["nb1"] * g
    v = F["b2"] * v + F["nb2"] * (g * g)
    u = m / (torch.sqrt(v) * F["root"] + F["eps"])
    return p * F["decay"] - F["lr"] * u, m, v


def _adam_factors():
    a = ADAM
    return dict(b1=a["beta1"], nb1=1.0 - a["beta1"], b2=a["beta2"], nb2=1.0 - a["beta2"], eps=a["eps"],
                decay=1.0 - a["lr"] * a["weight_decay"], lr=a["lr"] / (1.0 - a["beta1"] ** a["step"]),
                root=1.0 / math.sqrt(1.0 - a["beta2"] ** a["step"]))


def _plain_norm(s, c):
    dt = s["x"].dtype
    x, w = s["x"].float(), s["w"].float()
    if c["way"] == "backward":
        gy, rstd = s["gy"].float(), s["rstd"][:, None]
        xh, gw = x * rstd, gy * w
        gx = rstd * (gw - xh * (gw * xh).mean(dim=1, keepdim=True))
        if s["r"] is not None:  # the gradient that reaches the sum from behind the block
            gx = gx + s["r"].float()
        return [gx.to(dt), (gy * xh).sum(dim=0)]
    t = x + s["r"].float() if s["r"] is not None else x
    total = [t.to(dt)] if s["r"] is not None else []
    if c["way"] == "rows_q8":
        v, rstd = t, torch.ones((c["rows"], 1), device=t.device)
    else:
        v, rstd = t * w, torch.rsqrt(t.square().mean(dim=1, keepdim=True) + EPS)
    if c["way"] == "forward":
        return [(t * rstd * w).to(dt), rstd.reshape(-1)] + total
    amax = v.abs().amax(dim=1, keepdim=True)
    inv = torch.where(amax >= 2.0 ** -120, torch.full_like(amax, 127.0) / amax, torch.zeros_like(amax))
    scale = amax * rstd / 127.0
    return [torch.round(v * inv) * scale, scale.reshape(-1)] + total


def _plain_matmul(s, c):
    dt = _type(c["dtype"])
    w = s["w"].float()
    wm = w.t() if c["transposed"] else w
    if c["way"] == "backward":
        gz = s["gy"].float()
        if s["z"] is not None:
            gz = gz * _act_grad(s["z"].float(), c["act"])
        x = s["x"].float()
        gw = gz.t() @ x if c["transposed"] else x.t() @ gz
        return [(gz @ wm.t()).to(dt), gw.to(dt)] + ([gz.sum(dim=0)] if c["bias"] else [])
    z = s["x"].float() @ wm
    if c["dtype"] == "q8":
        z = z * s["xs"][:, None] * s["ws"]
    if s["b"] is not None:
        z = z + s["b"].float()
    y = _act(z, c["act"])
    if s["r"] is not None:
        y = y + s["r"].float()
    return [y.to(dt), z.to(dt)] if c["way"] == "train" else [y.to(dt)]


def _plain_gated(s, c):
    dt = _type(c["dtype"])
    x, wg, wu = s["x"].float(), s["wg"].float(), s["wu"].float()
    if c["way"] == "backward":
        gh, g, u = s["gh"].float(), s["g"].float(), s["u"].float()
        gg, gu = gh * u * _act_grad(g, c["act"]), gh * _act(g, c["act"])
        return [(gg @ wg.t() + gu @ wu.t()).to(dt), (x.t() @ gg).to(dt), (x.t() @ gu).to(dt)]
    if c["dtype"] == "q8":
        g, u = (x @ wg.t()) * s["xs"][:, None] * s["wgs"], (x @ wu.t()) * s["xs"][:, None] * s["wus"]
    else:
        g, u = x @ wg, x @ wu
    h = (_act(g, c["act"]) * u).to(dt)
    return [h, g.to(dt), u.to(dt)] if c["way"] == "train" else [h]


def _plain_adamw(s, c):
    F = _adam_factors()
    ms, vs = [], []
    for i in range(len(s["p"])):  # a plain training loop takes its tensors one by one
        m, v = s["m"][i], s["v"][i]
        if c["bits"] == 8:
            m, v = _decode_m(m, s["ms"][i]), _decode_v(v, s["vs"][i])
        p, m, v = _adam_update(s["p"][i].float(), s["g"][i].float(), m, v, F)
        s["p"][i].copy_(p)
        if s["copy"] is not None:
            s["copy"][i].copy_(p)
        if c["bits"] == 8:
            for name, (code, scale) in (("m", _encode_m(m)), ("v", _encode_v(v))):
                s[name][i].copy_(code)
                s[name + "s"][i].copy_(scale)
            m, v = _decode_m(s["m"][i], s["ms"][i]), _decode_v(s["v"][i], s["vs"][i])
        else:
            m, v = s["m"][i].copy_(m), s["v"][i].copy_(v)
        ms.append(m)
        vs.append(v)
    return [s["p"], ms, vs] + ([s["copy"]] if s["copy"] is not None else [])


def _run_own(s, c):
    from paper_2002_09481_amd import binding as ax

    if c["op"] == "norm":
        if c["way"] == "backward":
            return list(ax.ax_rmsnorm_backward(s["gy"], s["x"], s["w"], s["rstd"], gsum=s["r"]))
        if c["way"] == "forward":
            y, total, rstd = ax.ax_rmsnorm(s["x"], s["w"], residual=s["r"], eps=EPS)
            return [y, rstd] + ([total] if total is not None else [])
        # (the values that the codes stand for come out of the same kernel)
        _, scales, total, values = ax.ax_rmsnorm_q8(s["x"], None if c["way"] == "rows_q8" else s["w"], residual=s["r"],
                                                    eps=EPS, normalize=c["way"] == "q8", values=True)
        return [values, scales] + ([total] if total is not None else [])
    if c["op"] == "matmul":
        if c["way"] == "backward":
            gx, gw, gb = ax.ax_matmul_backward(s["gy"], s["x"], s["w"], s["z"], act=c["act"], transposed=c["transposed"],
                                               gb_out=None if c["bias"] else False)
            return [gx, gw] + ([gb] if c["bias"] else [])
        if c["dtype"] == "q8":
            return [ax.ax_matmul_q8(s["x"], s["xs"], s["w"], s["ws"], bias=s["b"], residual=s["r"], act=c["act"])]
        y, z = ax.ax_matmul(s["x"], s["w"], bias=s["b"], residual=s["r"], act=c["act"], transposed=c["transposed"],
                            save=c["way"] == "train")
        return [y, z] if c["way"] == "train" else [y]
    if c["op"] == "gated":
        if c["way"] == "backward":
            return list(ax.ax_gated_backward(s["gh"], s["x"], s["wg"], s["wu"], s["g"], s["u"], act=c["act"]))
        if c["dtype"] == "q8":
            return [ax.ax_gated_q8(s["x"], s["xs"], s["wg"], s["wgs"], s["wu"], s["wus"], act=c["act"])]
        h, g, u = ax.ax_gated(s["x"], s["wg"], s["wu"], act=c["act"], save=c["way"] == "train")
        return [h, g, u] if c["way"] == "train" else [h]
    opt = s["opt"]
    opt.step(**ADAM)
    ms, vs = opt.states() if c["bits"] == 8 else (s["m"], s["v"])
    return [s["p"], list(ms), list(vs)] + ([s["copy"]] if s["copy"] is not None else [])


def run(state):
    c = state["case"]
    if own:
        return _run_own(state, c)
    return {"norm": _plain_norm, "matmul": _plain_matmul, "gated": _plain_gated, "adamw": _plain_adamw}[c["op"]](state, c)


# ---- what a pass cannot do without --------------------------------------------------------------


def work(case):
    c = case
    e = 4 if c["dtype"] == "f32" else 2
    if c["op"] == "norm":
        n, rows, cols = c["rows"] * c["cols"], c["rows"], c["cols"]
        if c["way"] == "backward":
            return {"bytes": n * e * (3 + c["residual"]) + cols * (e + 4) + rows * 4, "flops": 10 * n}
        b = n * e * (1 + 2 * c["residual"]) + cols * e * (c["way"] != "rows_q8") + rows * 4
        return {"bytes": b + n * (e if c["way"] == "forward" else 5), "flops": 6 * n}
    if c["op"] == "matmul":
        M, K, N = c["M"], c["K"], c["N"]
        if c["way"] == "backward":
            b = e * (2 * M * K + 2 * K * N + M * N * (1 + (c["act"] != "none"))) + 4 * N * c["bias"]
            return {"bytes": b, "flops": 4.0 * M * K * N}
        o = 1 if c["dtype"] == "q8" else e
        b = o * (M * K + K * N) + e * (M * N * (1 + c["residual"] + (c["way"] == "train")) + N * c["bias"])
        return {"bytes": b + (4 * (M + N) if c["dtype"] == "q8" else 0), "flops": 2.0 * M * K * N}
    if c["op"] == "gated":
        M, K, F = c["M"], c["K"], c["F"]
        if c["way"] == "backward":
            return {"bytes": e * (3 * M * F + 2 * M * K + 4 * K * F), "flops": 8.0 * M * K * F}
        o = 1 if c["dtype"] == "q8" else e
        b = o * (M * K + 2 * K * F) + e * M * F * (3 if c["way"] == "train" else 1)
        return {"bytes": b + (4 * (M + 2 * F) if c["dtype"] == "q8" else 0), "flops": 4.0 * M * K * F}
    n = sum(math.prod(sh) for sh in _tensor_shapes(c))
    b = {"f32": 12, "mixed": 12, "bf16": 6}[c["dtype"]]  # parameters read and written, gradients, 16-bit copies
    state = 16 if c["bits"] == 32 else 4 + 16.0 / BLOCK + 8  # (8 bits: the values the states stand for are written too)
    return {"bytes": n * (b + state), "flops": 15 * n}


# ---- the definition in 64 bits ------------------------------------------------------------------


def exact(case, seed):
    c = case
    if c["op"] == "adamw" and sum(math.prod(sh) for sh in _tensor_shapes(c)) > 4e8:
        return None
    s = prepare(c, seed)
    d = lambda t: None if t is None else t.double()  # noqa: E731

    def act(z):
        if c["act"] == "silu":
            return z * torch.special.expit(z)
        if c["act"] == "gelu":
            return z * torch.special.ndtr(z)
        return torch.relu(z) if c["act"] == "relu" else z

    def slope(z):
        if c["act"] == "silu":
            e = torch.special.expit(z)
            return e + z * e * torch.special.expit(-z)
        if c["act"] == "gelu":
            return torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
        return torch.heaviside(z, torch.zeros((), dtype=z.dtype, device=z.device)) if c["act"] == "relu" else torch.ones_like(z)

    if c["op"] == "norm":
        x, w, r = d(s["x"]), d(s["w"]), d(s["r"])
        if c["way"] == "backward":
            k, gy = d(s["rstd"])[:, None], d(s["gy"])
            gx = k * gy * w - k ** 3 * x * torch.sum(gy * w * x, dim=1, keepdim=True) / c["cols"]
            return [gx if r is None else gx + r, torch.sum(gy * x * k, dim=0)]
        t = x if r is None else x + r
        total = [] if r is None else [t]
        rms = torch.sqrt((t ** 2).mean(dim=1) + EPS)
        if c["way"] == "forward":
            return [t / rms[:, None] * w, 1.0 / rms] + total
        y = t if c["way"] == "rows_q8" else t / rms[:, None] * w
        top = torch.amax(torch.abs(y), dim=1)
        step = torch.where(top > 0, top, torch.ones_like(top)) / 127.0
        return [torch.round(y / step[:, None]) * (top / 127.0)[:, None], top / 127.0] + total
    if c["op"] == "matmul":
        x, w, b, r = d(s["x"]), d(s["w"]), d(s["b"]), d(s["r"])
        if c["dtype"] == "q8":
            x, w = x * d(s["xs"])[:, None], w * d(s["ws"])[:, None]
        w = w.T.contiguous() if c["transposed"] else w
        if c["way"] == "backward":
            gz = d(s["gy"]) * (1.0 if s["z"] is None else slope(d(s["z"])))
            gw = torch.matmul(x.T, gz)
            return [torch.matmul(gz, w.T), gw.T if c["transposed"] else gw] + ([gz.sum(dim=0)] if c["bias"] else [])
        z = torch.matmul(x, w)
        z = z if b is None else z + b
        y = act(z) if r is None else act(z) + r
        return [y, z] if c["way"] == "train" else [y]
    if c["op"] == "gated":
        x, wg, wu = d(s["x"]), d(s["wg"]), d(s["wu"])
        if c["dtype"] == "q8":
            x = x * d(s["xs"])[:, None]
            wg, wu = (wg * d(s["wgs"])[:, None]).T, (wu * d(s["wus"])[:, None]).T
        if c["way"] == "backward":
            gh, g, u = d(s["gh"]), d(s["g"]), d(s["u"])
            gg, gu = gh * u * slope(g), gh * act(g)
            return [torch.matmul(gg, wg.T) + torch.matmul(gu, wu.T), torch.matmul(x.T, gg), torch.matmul(x.T, gu)]
        g, u = torch.matmul(x, wg), torch.matmul(x, wu)
        h = act(g) * u
        return [h, g, u] if c["way"] == "train" else [h]
    a, out = ADAM, [[], [], []]

    def blocks(t, fill):
        n = t.numel()
        return torch.nn.functional.pad(t.reshape(-1), (0, -n % BLOCK), value=fill).view(-1, BLOCK)

    for i, p in enumerate(s["p"]):
        p, g, m, v = d(p), d(s["g"][i]), d(s["m"][i]), d(s["v"][i])
        if c["bits"] == 8:
            n = m.numel()
            m = (torch.sign(blocks(m, 0)) * (blocks(m, 0) / 127) ** 2 * d(s["ms"][i])[:, None]).reshape(-1)[:n].view(p.shape)
            v = ((blocks(v, 0) / 255) ** 4 * d(s["vs"][i])[:, None]).reshape(-1)[:n].view(p.shape)
        m = a["beta1"] * m + (1 - a["beta1"]) * g
        v = a["beta2"] * v + (1 - a["beta2"]) * g ** 2
        mh, vh = m / (1 - a["beta1"] ** a["step"]), v / (1 - a["beta2"] ** a["step"])
        out[0].append(p * (1 - a["lr"] * a["weight_decay"]) - a["lr"] * mh / (torch.sqrt(vh) + a["eps"]))
        if c["bits"] == 8:  # the states as they are kept
            top = blocks(m, 0).abs().amax(dim=1, keepdim=True)
            code = torch.round(127 * torch.sqrt(blocks(m, 0).abs() / top))
            m = (torch.sign(blocks(m, 0)) * (code / 127) ** 2 * top).reshape(-1)[:n].view(p.shape)
            top = blocks(v, 0).amax(dim=1, keepdim=True)
            code = torch.round(255 * (blocks(v, 0) / top) ** 0.25).clamp(min=1)
            v = ((code / 255) ** 4 * top).reshape(-1)[:n].view(p.shape)
        out[1].append(m)
        out[2].append(v)
    return out + ([out[0]] if c["dtype"] == "mixed" else [])
