"""Performance cases of the operators of a feed-forward block made of experts, and of its weights in 4 bits.

Every case is a dict of plain values; "op" names the operator and "way" the direction:

  route    the router's choice: each token's k experts with their weights, and the order of rows by expert
             forward    experts, weights, the experts' offsets, every choice's row, every row's token
             backward   the gradient of the logits from that of the weights
  experts  rows grouped by expert, at ragged sizes, times the matrix of their expert; "gated": the pair of
           projections act(x wg) * (x wu), otherwise one product
             serve      the output alone
             train      the output and what the backward pass needs
             backward   gradients of the rows and of the weights
  combine  every token's sum of its experts' rows with the router's weights, and the residual
             forward / backward (gradients of the rows and of the weights)
  q4       products with weights of 4 bits and a scale for each group of a row, "gated" as above; with
           "experts" above one the rows are grouped by expert (forward only)

"dtype" is the operands' type, "f32" or "bf16".  Where `own` is false the operators are computed in their
plain form, elementary torch operations in 32 bits; where it is true, by this library's entry points.
"""

import math

import torch

own = False

DEV = "cuda" if torch.cuda.is_available() else "cpu"

MOST_TERMS = 2 * 8192 * 2048 * 8192  # rows * inputs * outputs of a product by experts
MOST_WEIGHTS = 8 * 2048 * 8192  # elements of one weight, over all experts
MOST_ELEMS = 2 * 8192 * 4096  # of the rows that are combined


def listed():
    return [
        # one token being decoded, many small experts: nothing but latency
        dict(name="route_token", op="route", way="forward", tokens=1, experts=64, k=6, dtype="bf16", normalize=True),
        # the tokens of a training step
        dict(name="route_batch", op="route", way="forward", tokens=16384, experts=128, k=8, dtype="bf16", normalize=True),
        # the router's gradient, weights out of the softmax over all experts, odd sizes
        dict(name="route_backward_odd", op="route", way="backward", tokens=6007, experts=60, k=4, dtype="f32", normalize=False),
        # a few sequences decoded together: most experts see a row or none
        dict(name="experts_decode", op="experts", way="serve", gated=False, tokens=5, k=4, experts=64, K=1408, N=2048,
             dtype="bf16", act="none", transposed=False),
        # the largest training step: few large experts
        dict(name="experts_gated_train", op="experts", way="train", gated=True, tokens=8192, k=2, experts=8, K=2048, N=8192,
             dtype="bf16", act="silu", transposed=False),
        # gradients with many experts of ragged sizes
        dict(name="experts_gated_backward", op="experts", way="backward", gated=True, tokens=2047, k=4, experts=32, K=1024,
             N=1416, dtype="bf16", act="silu", transposed=False),
        # gradients of a float32 network, odd sizes
        dict(name="experts_backward_f32", op="experts", way="backward", gated=False, tokens=1531, k=2, experts=5, K=512, N=1000,
             dtype="f32", act="gelu", transposed=False),
        # back into the residual stream behind a training step's experts: bandwidth
        dict(name="combine_large", op="combine", way="forward", tokens=8192, k=2, cols=4096, dtype="bf16", residual=True),
        # its gradients for an odd number of tokens
        dict(name="combine_backward_odd", op="combine", way="backward", tokens=3001, k=4, cols=1000, dtype="bf16",
             residual=False),
        # a projection for one token: every weight is read once, for one row
        dict(name="q4_token", op="q4", gated=False, tokens=1, k=1, experts=1, K=4096, N=4096, group=128, dtype="bf16",
             act="none", bias=True, residual=True),
        # the experts' projections for a few sequences decoded together, odd width
        dict(name="q4_gated_experts", op="q4", gated=True, tokens=17, k=4, experts=32, K=2048, N=1409, group=32, dtype="bf16",
             act="silu", bias=False, residual=False),
        # a prompt through the same kind of weights
        dict(name="q4_prompt", op="q4", gated=False, tokens=1027, k=1, experts=1, K=4096, N=4096, group=64, dtype="bf16",
             act="gelu", bias=True, residual=False),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm; every other one is made odd."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(lo, min(hi, n | 1 if rng.random() < 0.5 else -(-n // 8) * 8))


def draw(rng):
    op = rng.choice(["route", "experts", "combine", "q4"])
    k = rng.choice([1, 2, 2, 3, 4, 6, 8])
    if op == "route":
        return dict(op=op, way=rng.choice(["forward", "backward"]), tokens=_log(rng, 1, 16384), experts=_log(rng, 8, 256), k=k,
                    dtype=rng.choice(["bf16", "f32"]), normalize=rng.random() < 0.5)
    if op == "combine":
        cols = _log(rng, 64, 8192)
        return dict(op=op, way=rng.choice(["forward", "backward"]), tokens=_log(rng, 1, min(16384, MOST_ELEMS // 2 // (cols * k))),
                    k=k, cols=cols, dtype=rng.choice(["bf16", "f32"]), residual=rng.random() < 0.5)
    if op == "experts":
        way = rng.choice(["serve", "train", "backward"])
        E = max(k, _log(rng, 2, 64))
        K = _log(rng, 64, 4096)
        N = _log(rng, 64, min(4096, MOST_WEIGHTS // 2 // (E * K)))
        most = min(16384, MOST_TERMS // 4 // (K * N))
        gated = rng.random() < 0.5
        return dict(op=op, way=way, gated=gated, tokens=_log(rng, 1, 32 if way == "serve" and rng.random() < 0.5 else most // k),
                    k=k, experts=E, K=K, N=N, dtype=rng.choice(["bf16", "f32"]),
                    act=rng.choice(["relu", "silu", "gelu"] + ["none"] * (not gated)), transposed=not gated and rng.random() < 0.5)
    E = 1 if rng.random() < 0.5 else max(k, _log(rng, 2, 32))
    K = _log(rng, 64, 8192)
    N = _log(rng, 64, min(8192, MOST_WEIGHTS // (E * K)))
    gated = rng.random() < 0.4
    return dict(op=op, gated=gated, tokens=_log(rng, 1, 64 if rng.random() < 0.5 else 2048 // (k if E > 1 else 1)),
                k=k if E > 1 else 1, experts=E, K=K, N=N, group=rng.choice([32, 64, 128]), dtype=rng.choice(["bf16", "f32"]),
                act=rng.choice(["relu", "silu", "gelu"] + ["none"] * (not gated)), bias=E == 1 and not gated and rng.random() < 0.5,
                residual=E == 1 and not gated and rng.random() < 0.5)


# ---- inputs, made from the seed ---------------------------------------------------------------


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 7919 + 29)
    return g


def _type(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _randn(g, shape, scale, dtype):
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)


def _logits(g, c):
    """A router's logits: some experts are liked more than others by all tokens."""
    E = c["experts"]
    return torch.randn((c["tokens"], E), generator=g, device=DEV) + 0.7 * torch.randn((E,), generator=g, device=DEV)


def _grouping(g, c):
    """Tokens of the rows in the order of their experts, the experts' offsets, and the sizes as the host's numbers."""
    experts = torch.sort(_logits(g, c), dim=1, descending=True, stable=True).indices[:, : c["k"]].reshape(-1)
    by_expert, order = torch.sort(experts, stable=True)
    offsets = torch.searchsorted(by_expert, torch.arange(c["experts"] + 1, device=DEV)).to(torch.int32)
    return (order // c["k"]).to(torch.int32), offsets, offsets.tolist()


def _quantized(g, rows, cols, group):
    """Weights of 4 bits: two codes of -8 .. 7 (plus eight) a byte, the even column's in the low half, and bf16 scales."""
    n = -(-cols // group)
    w = torch.randn((rows, n * group), generator=g, device=DEV) / math.sqrt(cols)
    w[:, cols:] = 0.0
    w = w.view(rows, n, group)
    scales = (w.abs().amax(dim=2) / 7.0).to(torch.bfloat16)
    codes = torch.round(w / scales.float()[:, :, None]).clamp(-8, 7).view(rows, -1)[:, : cols + cols % 2].to(torch.int8)
    u = (codes + 8).to(torch.uint8)
    return u[:, 0::2] | (u[:, 1::2] << 4), scales


def _unpacked(packed, cols):
    """Codes -8 .. 7 of nibbles."""
    return (torch.stack((packed & 15, packed >> 4), dim=-1).view(*packed.shape[:-1], -1)[..., :cols].to(torch.int8)) - 8


def prepare(case, seed):
    c, g = case, _gen(seed)
    s = {"case": c}
    dt = _type(c["dtype"])
    if c["op"] == "route":
        s["logits"] = _logits(g, c).to(dt)
        if c["way"] == "backward":
            s["e"], s["w"] = _plain_choice(s["logits"], c)
            s["gw"] = _randn(g, (c["tokens"], c["k"]), 0.1, torch.float32)
        return s
    T, k = c["tokens"], c["k"]
    if c["op"] == "combine":
        n = T * k
        s["h"] = _randn(g, (n, c["cols"]), 1.0, dt)
        s["rows"] = torch.randperm(n, generator=g, device=DEV).to(torch.int32).view(T, k)
        s["w"] = torch.softmax(torch.randn((T, k), generator=g, device=DEV), dim=1)
        s["r"] = _randn(g, (T, c["cols"]), 1.0, dt) if c["residual"] else None
        if c["way"] == "backward":
            s["gy"] = _randn(g, (T, c["cols"]), 0.02, dt)
        return s
    E, K, N = c["experts"], c["K"], c["N"]
    s["x"] = _randn(g, (T, K), 1.0, dt)
    if E > 1:
        s["tokens"], s["offsets"], s["sizes"] = _grouping(g, c)
    if c["op"] == "experts":
        shape = (E, N, K) if c["transposed"] else (E, K, N)
        names = ("wg", "wu") if c["gated"] else ("w",)
        for n in names:
            s[n] = _randn(g, shape, 1.0 / math.sqrt(K), dt)
        if c["way"] == "backward":
            s["gy"] = _randn(g, (T * k, N), 0.02, dt)
            if c["gated"] or c["act"] != "none":
                s["z"] = _randn(g, (T * k, N), 1.0, dt)
            if c["gated"]:
                s["u"] = _randn(g, (T * k, N), 1.0, dt)
        return s
    for n in ("wg", "wu") if c["gated"] else ("w",):
        packed, scales = _quantized(g, E * N, K, c["group"])
        if own:  # the weights as a program keeps them, laid out once
            from paper_2002_09481_amd import binding as ax

            s[n] = ax.ax_pack_q4(_unpacked(packed, K).view(E, N, K), scales.view(E, N, -1), group=c["group"])
        else:
            s[n] = packed.view(E, N, -1), scales.view(E, N, -1)
    s["b"] = _randn(g, (N,), 0.5, dt) if c["bias"] else None
    s["r"] = _randn(g, (T, N), 1.0, dt) if c["residual"] else None
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


def _plain_choice(logits, c):
    """The k largest logits of each row, ties to the lowest index, and the softmax over them or over all."""
    top, idx = torch.sort(logits.float(), dim=1, descending=True, stable=True)
    e = torch.exp(top - top[:, :1])
    w = e[:, : c["k"]] / (e[:, : c["k"]] if c["normalize"] else e).sum(dim=1, keepdim=True)
    return idx[:, : c["k"]].to(torch.int32).contiguous(), w


def _plain_route(s, c):
    if c["way"] == "backward":
        e, gw, w = s["e"].long(), s["gw"], s["w"]
        inner = (gw * w).sum(dim=1, keepdim=True)
        if c["normalize"]:
            full = torch.zeros_like(s["logits"], dtype=torch.float32).scatter_(1, e, w * (gw - inner))
        else:
            x = s["logits"].float()
            p = torch.exp(x - x.amax(dim=1, keepdim=True))
            p = p / p.sum(dim=1, keepdim=True)
            full = p * (torch.zeros_like(x).scatter_(1, e, gw) - inner)
        return [full.to(s["logits"].dtype)]
    experts, w = _plain_choice(s["logits"], c)
    by_expert, order = torch.sort(experts.reshape(-1), stable=True)
    offsets = torch.searchsorted(by_expert, torch.arange(c["experts"] + 1, device=order.device, dtype=torch.int32))
    rows = torch.empty_like(order).scatter_(0, order, torch.arange(order.numel(), device=order.device))
    return [experts, w, offsets.to(torch.int32), rows.view(experts.shape).to(torch.int32), (order // c["k"]).to(torch.int32)]


def _each(s, c):
    """The experts that have rows: expert, first row, last."""
    o = s["sizes"]
    return [(e, o[e], o[e + 1]) for e in range(c["experts"]) if o[e + 1] > o[e]]


def _plain_experts(s, c):
    dt = s["x"].dtype
    x = s["x"].float()[s["tokens"].long()]
    n = x.shape[0]
    names = ("wg", "wu") if c["gated"] else ("w",)
    new = lambda width: torch.empty((n, width), dtype=torch.float32, device=x.device)  # noqa: E731
    if c["way"] != "backward":
        z = [new(c["N"]) for _ in names]
        for e, a, b in _each(s, c):
            for out, name in zip(z, names):
                w = s[name][e].float()
                torch.matmul(x[a:b], w.t() if c["transposed"] else w, out=out[a:b])
        y = _act(z[0], c["act"])
        if c["gated"]:
            y = y * z[1]
        train = c["way"] == "train" and (c["gated"] or c["act"] != "none")
        return [y.to(dt)] + ([t.to(dt) for t in z] if train else [])
    gy = s["gy"].float()
    if c["gated"]:
        z, u = s["z"].float(), s["u"].float()
        gz = [gy * u * _act_grad(z, c["act"]), gy * _act(z, c["act"])]
    else:
        gz = [gy * _act_grad(s["z"].float(), c["act"]) if c["act"] != "none" else gy]
    gx, gw = new(c["K"]), [torch.zeros_like(s[name]) for name in names]
    for e, a, b in _each(s, c):
        total = 0.0
        for g, out, name in zip(gz, gw, names):
            w = s[name][e].float()
            total = total + g[a:b] @ (w if c["transposed"] else w.t())
            out[e] = g[a:b].t() @ x[a:b] if c["transposed"] else x[a:b].t() @ g[a:b]
        gx[a:b] = total
    return [gx.to(dt)] + gw


def _plain_combine(s, c):
    rows, w = s["rows"].long(), s["w"]
    if c["way"] == "backward":
        gy = s["gy"].float()
        gh = torch.empty_like(s["h"])
        gh[rows.reshape(-1)] = (w[:, :, None] * gy[:, None, :]).to(gh.dtype).view(-1, c["cols"])
        return [gh, (s["h"][rows].float() * gy[:, None, :]).sum(dim=2)]
    y = (w[:, :, None] * s["h"][rows].float()).sum(dim=1)
    return [(y if s["r"] is None else y + s["r"].float()).to(s["h"].dtype)]


def _plain_q4(s, c):
    x = s["x"].float()
    names = ("wg", "wu") if c["gated"] else ("w",)

    def weight(name, e):
        packed, scales = s[name]
        v = _unpacked(packed[e], c["K"]).float()
        return v * scales[e].float().repeat_interleave(c["group"], dim=1)[:, : c["K"]]

    if c["experts"] == 1:
        z = [x @ weight(name, 0).t() for name in names]
    else:
        x = x[s["tokens"].long()]
        z = [torch.empty((x.shape[0], c["N"]), dtype=torch.float32, device=x.device) for _ in names]
        for e, a, b in _each(s, c):
            for out, name in zip(z, names):
                torch.matmul(x[a:b], weight(name, e).t(), out=out[a:b])
    if s["b"] is not None:
        z[0] = z[0] + s["b"].float()
    y = _act(z[0], c["act"])
    if c["gated"]:
        y = y * z[1]
    if s["r"] is not None:
        y = y + s["r"].float()
    return [y.to(s["x"].dtype)]


def _run_own(s, c):
    from paper_2002_09481_amd import binding as ax

    if c["op"] == "route":
        if c["way"] == "backward":
            return [ax.ax_route_backward(s["gw"], s["logits"], s["e"], s["w"], normalize=c["normalize"])]
        return list(ax.ax_route(s["logits"], c["k"], normalize=c["normalize"]))
    if c["op"] == "combine":
        if c["way"] == "backward":
            return list(ax.ax_combine_backward(s["gy"], s["h"], s["rows"], s["w"]))
        return [ax.ax_combine(s["h"], s["rows"], s["w"], residual=s["r"])]
    group = dict(offsets=s["offsets"], tokens=s["tokens"]) if c["experts"] > 1 else {}
    if c["op"] == "q4":
        if c["gated"]:
            return [ax.ax_gated_q4(s["x"], s["wg"], s["wu"], act=c["act"], **group)]
        return [ax.ax_matmul_q4(s["x"], s["w"], bias=s["b"], residual=s["r"], act=c["act"], **group)]
    if c["gated"]:
        if c["way"] == "backward":
            return list(ax.ax_gated_experts_backward(s["gy"], s["x"], s["wg"], s["wu"], s["z"], s["u"], act=c["act"], **group))
        h, g, u = ax.ax_gated_experts(s["x"], s["wg"], s["wu"], act=c["act"], save=c["way"] == "train", **group)
        return [h, g, u] if c["way"] == "train" else [h]
    if c["way"] == "backward":
        return list(ax.ax_matmul_experts_backward(s["gy"], s["x"], s["w"], z=s.get("z"), act=c["act"], transposed=c["transposed"],
                                                  **group))
    y, z = ax.ax_matmul_experts(s["x"], s["w"], act=c["act"], transposed=c["transposed"],
                                save=c["way"] == "train" and c["act"] != "none", **group)
    return [y] if z is None else [y, z]


def run(state):
    c = state["case"]
    if own:
        return _run_own(state, c)
    return {"route": _plain_route, "experts": _plain_experts, "combine": _plain_combine, "q4": _plain_q4}[c["op"]](state, c)


# ---- what a pass cannot do without --------------------------------------------------------------


def work(case):
    c = case
    e = 4 if c["dtype"] == "f32" else 2
    T, k = c["tokens"], c["k"]
    if c["op"] == "route":
        E = c["experts"]
        if c["way"] == "backward":
            return {"bytes": T * E * e * (1 if c["normalize"] else 2) + T * k * 12, "flops": 6 * T * E}
        return {"bytes": T * E * e + T * k * 16 + (E + 1) * 4, "flops": 4 * T * E}
    if c["op"] == "combine":
        n = T * c["cols"]
        if c["way"] == "backward":
            return {"bytes": n * e * (1 + 2 * k) + T * k * 12, "flops": 3 * n * k}
        return {"bytes": n * e * (k + 1 + c["residual"]) + T * k * 8, "flops": 2 * n * k}
    E, K, N = c["experts"], c["K"], c["N"]
    R, nw = T * k, 2 if c["gated"] else 1
    used = min(E, R)
    if c["op"] == "q4":
        b = used * nw * N * (K * 0.5 + 2 * -(-K // c["group"])) + e * (T * K + R * N * (1 + c["residual"]) + N * c["bias"])
        return {"bytes": b, "flops": 2.0 * nw * R * K * N}
    w = used * nw * K * N * e
    if c["way"] == "backward":
        kept = 3 if c["gated"] else 1 + (c["act"] != "none")
        return {"bytes": w + E * nw * K * N * e + e * (R * N * kept + T * K + R * K), "flops": 4.0 * nw * R * K * N}
    outs = 1 + (c["way"] == "train") * (2 if c["gated"] else int(c["act"] != "none"))
    return {"bytes": w + e * (T * K + R * N * outs), "flops": 2.0 * nw * R * K * N}


# ---- the definition in 64 bits ------------------------------------------------------------------


def exact(case, seed):
    global own
    kept, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    c = case
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

    if c["op"] == "route":
        x = d(s["logits"])
        p = torch.softmax(x, dim=1)
        if c["way"] == "backward":
            hot = torch.nn.functional.one_hot(s["e"].long(), c["experts"]).double()
            w, gw = d(s["w"]), d(s["gw"])
            if c["normalize"]:  # (through the weights that the forward pass left)
                return [torch.einsum("tke,tk->te", hot, w * gw) - torch.einsum("tke,tk->te", hot, w) * (w * gw).sum(1, keepdim=True)]
            g = torch.einsum("tke,tk->te", hot, gw)
            return [p * g - p * (w * gw).sum(1, keepdim=True)]
        left, chosen, at = x.clone(), [], torch.arange(c["experts"], device=x.device)
        for _ in range(c["k"]):
            best = torch.where(left == left.amax(dim=1, keepdim=True), at, c["experts"]).amin(dim=1)
            chosen.append(best)
            left[torch.arange(len(best), device=x.device), best] = -math.inf
        chosen = torch.stack(chosen, dim=1)
        w = torch.gather(p, 1, chosen)
        if c["normalize"]:
            w = w / w.sum(dim=1, keepdim=True)
        hot = torch.nn.functional.one_hot(chosen.reshape(-1), c["experts"])
        ends = hot.sum(dim=0).cumsum(0)
        first = torch.cat((ends.new_zeros(1), ends))
        rank = (hot.cumsum(dim=0) * hot).sum(dim=1) - 1
        rows = first[chosen.reshape(-1)] + rank
        tokens = torch.zeros_like(rows)
        tokens[rows] = torch.arange(rows.numel(), device=rows.device) // c["k"]
        i = lambda t: t.to(torch.int32)  # noqa: E731
        return [i(chosen), w, i(first), i(rows).view(chosen.shape), i(tokens)]
    if c["op"] == "combine":
        h, w, rows = d(s["h"]), d(s["w"]), s["rows"].long()
        if c["way"] == "backward":
            gy = d(s["gy"])
            gh = torch.zeros_like(h)
            gw = torch.zeros_like(w)
            for j in range(c["k"]):
                gh[rows[:, j]] = gy * w[:, j : j + 1]
                gw[:, j] = torch.linalg.vecdot(gy, h[rows[:, j]])
            return [gh, gw]
        y = torch.zeros((c["tokens"], c["cols"]), dtype=torch.float64, device=h.device) if s["r"] is None else d(s["r"])
        for j in range(c["k"]):
            y = y + h[rows[:, j]] * w[:, j : j + 1]
        return [y]
    E, K, N = c["experts"], c["K"], c["N"]
    names = ("wg", "wu") if c["gated"] else ("w",)
    R = c["tokens"] * c["k"]
    expert = torch.zeros(R, dtype=torch.long, device=s["x"].device)
    token = torch.arange(R, device=expert.device)
    if E > 1:
        token = s["tokens"].long()
        expert = torch.searchsorted(s["offsets"].long(), torch.arange(R, device=expert.device), right=True) - 1
    x = d(s["x"])[token]

    def weight(name, e):  # [K, N]
        if c["op"] == "q4":
            packed, scales = s[name]
            v = torch.empty((N, 2 * packed.shape[2]), dtype=torch.float64, device=x.device)
            v[:, 0::2], v[:, 1::2] = (packed[e] % 16).double() - 8, (packed[e] // 16).double() - 8
            col = torch.arange(K, device=x.device) // c["group"]
            return (v[:, :K] * scales[e].double()[:, col]).T
        return d(s[name][e]).T if c["transposed"] else d(s[name][e])

    if c.get("way") == "backward":
        gy = d(s["gy"])
        if c["gated"]:
            gz = [gy * d(s["u"]) * slope(d(s["z"])), gy * act(d(s["z"]))]
        else:
            gz = [gy * (slope(d(s["z"])) if c["act"] != "none" else 1.0)]
        gx = torch.zeros((R, K), dtype=torch.float64, device=x.device)
        gw = [torch.zeros(tuple(s[n].shape), dtype=torch.float64, device=x.device) for n in names]
        for e in range(E):
            at = torch.nonzero(expert == e).reshape(-1)
            for g, out, name in zip(gz, gw, names):
                gx[at] += torch.matmul(g[at], weight(name, e).T.contiguous())
                t = torch.matmul(x[at].T, g[at])
                out[e] = t.T if c["transposed"] else t
        return [gx] + gw
    z = [torch.zeros((R, N), dtype=torch.float64, device=x.device) for _ in names]
    for e in range(E):
        at = torch.nonzero(expert == e).reshape(-1)
        for out, name in zip(z, names):
            out[at] = torch.matmul(x[at], weight(name, e).contiguous())
    if s.get("b") is not None:
        z[0] = z[0] + d(s["b"])
    y = act(z[0])
    if c["gated"]:
        y = y * z[1]
    if s.get("r") is not None:
        y = y + d(s["r"])
    train = c.get("way") == "train" and (c["gated"] or c["act"] != "none")
    return [y] + (z if train else [])
