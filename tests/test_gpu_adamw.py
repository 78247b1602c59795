"""The AdamW step over many tensors: bit for bit the stated float32 operations (numpy), near the definition in 64 bits."""

import numpy as np
import pytest
import torch

import ff_common as F
from paper_2002_09481_amd import binding as ax

pytestmark = pytest.mark.gpu
f4 = np.float32
HYPER = dict(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.05)
# empty, one element, odd, around the blocks of 256 and the workgroups' 4096
SIZES = [0, 1, 5, 255, 256, 257, 1000, 4095, 4096, 4097, 20001]


def encode(x, top, power, levels):
    """Codes and scales of one tensor's blocks: float32 operations, one at a time."""
    n = x.size
    b = np.pad(x, (0, -n % 256)).reshape(-1, 256)
    scale = np.abs(b).max(axis=1)
    with np.errstate(divide="ignore"):
        inv = np.where(scale >= f4(2.0 ** -126), f4(1) / scale, f4(0)).astype(f4)[:, None]
    r = np.abs(b) * inv
    for _ in range(power):
        r = np.sqrt(r)
    c = np.rint(r * f4(levels))
    if power == 2:
        c = np.where((b > 0) & (inv > 0), np.maximum(c, 1), c)
    return np.where(b < 0, -c, c).reshape(-1)[:n].astype(top), scale


def decode(c, scale, levels):
    r = c.astype(f4) * f4(1.0 / levels)
    s = np.repeat(scale, 256)[:c.size]
    if levels == 127:
        return r * np.abs(r) * s
    r = r * r
    return r * r * s


def step_of(p, g, m, v, h, step, gs=None):
    g = g if gs is None else g * f4(gs)
    m = f4(h["beta1"]) * m + f4(1 - h["beta1"]) * g
    v = f4(h["beta2"]) * v + f4(1 - h["beta2"]) * (g * g)
    u = m / (np.sqrt(v) * f4(1 / np.sqrt(1 - h["beta2"] ** step)) + f4(h["eps"]))
    return p * f4(1 - h["lr"] * h["weight_decay"]) - f4(h["lr"] / (1 - h["beta1"] ** step)) * u, m, v


def _make(sizes, pdt, gdt, seed):
    g = F.gen(seed)
    return ([F.randn(g, (n,), 0.1, pdt).cuda() for n in sizes], [F.randn(g, (n,), 0.01, gdt).cuda() for n in sizes])


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("pdt,gdt", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f32")])
def test_steps(pdt, gdt, bits):
    P, G = _make(SIZES, F.DT[pdt], F.DT[gdt], 1)
    copies = [torch.zeros_like(p, dtype=torch.bfloat16) for p in P]
    opt = ax.AxAdamW(P, G, copies=copies, bits=bits)
    ref = [(p.cpu().float().numpy(), np.zeros(p.numel(), f4), np.zeros(p.numel(), f4)) for p in P]
    far = [(p.cpu().double(), torch.zeros(p.numel(), dtype=torch.float64), torch.zeros(p.numel(), dtype=torch.float64)) for p in P]
    for k in range(1, 4):
        if k > 1:
            G = _make(SIZES, F.DT[pdt], F.DT[gdt], k)[1]
            opt.set_grads(G)
        opt.step(step=k, **HYPER)
        ms, vs = opt.states()
        for i, n in enumerate(SIZES):
            g = G[i].cpu().float().numpy()
            p, m, v = step_of(*ref[i][:1], g, *ref[i][1:], HYPER, k)
            if bits == 8 and n:
                (cm, sm), (cv, sv) = encode(m, np.int8, 1, 127), encode(v, np.uint8, 2, 255)
                assert np.array_equal(opt.m[i].cpu().numpy(), cm) and np.array_equal(opt.v[i].cpu().numpy(), cv)
                assert np.array_equal(opt.m_scales[i].cpu().numpy(), sm) and np.array_equal(opt.v_scales[i].cpu().numpy(), sv)
                m, v = decode(cm, sm, 127), decode(cv, sv, 255)
            p = torch.from_numpy(p.astype(f4)).to(F.DT[pdt])
            assert torch.equal(P[i].cpu(), p)
            assert torch.equal(ms[i].cpu(), torch.from_numpy(m)) and torch.equal(vs[i].cpu(), torch.from_numpy(v))
            ref[i] = (p.float().numpy(), m, v)
            if bits == 32 and pdt == "f32":  # the definition
                gd, (pd, md, vd) = G[i].cpu().double(), far[i]
                md, vd = 0.9 * md + (1 - 0.9) * gd, 0.99 * vd + (1 - 0.99) * gd ** 2
                upd = HYPER["lr"] * (md / (1 - 0.9 ** k)) / (torch.sqrt(vd / (1 - 0.99 ** k)) + 1e-8)
                far[i] = (pd * (1 - HYPER["lr"] * 0.05) - upd, md, vd)
                # each step rounds p a few times; m may cancel, at most to the size of its terms: 0.04 / sqrt(v) of them
                F.assert_within(P[i], far[i][0], k * 4 * F.U * (pd.abs() + 0.1) + k * 64 * F.U * HYPER["lr"] * 10)
    for p, c, n in zip(P, copies, SIZES):
        if n:
            assert torch.equal(c, p.to(torch.bfloat16))


def test_more_tensors_than_one_launch_takes():
    sizes = [(i * 37) % 700 for i in range(131)]
    P, G = _make(sizes, torch.float32, torch.float32, 3)
    want = [torch.from_numpy(step_of(p.cpu().numpy(), g.cpu().numpy(), np.zeros(p.numel(), f4), np.zeros(p.numel(), f4), HYPER, 1)[0])
            for p, g in zip(P, G)]
    ax.AxAdamW(P, G).step(step=1, **HYPER)
    assert all(torch.equal(p.cpu(), w) for p, w in zip(P, want))


@pytest.mark.parametrize("bits", [32, 8])
def test_views_at_any_element(bits):
    """Tensors that start off their vectors' alignment, next to memory that is not theirs."""
    n, off = 1003, 3
    make = lambda dt, k: torch.full((k + 2 * off,), 5, dtype=dt, device="cuda")  # noqa: E731
    P, G = _make([n], torch.bfloat16, torch.float32, 5)
    want = ax.AxAdamW([P[0].clone()], G, bits=bits)
    want.step(step=1, **HYPER)
    mt, vt = (torch.int8, torch.uint8) if bits == 8 else (torch.float32, torch.float32)
    bufs = [make(torch.bfloat16, n), make(torch.float32, n), make(mt, n), make(vt, n), make(torch.bfloat16, n)]
    p, g, m, v, c = (b[off:off + n] for b in bufs)
    p.copy_(P[0]), g.copy_(G[0]), m.zero_(), v.zero_()
    scales = [torch.zeros(4, device="cuda") for _ in range(2)] if bits == 8 else [None, None]
    opt = ax.AxAdamW([p], [g], [m], [v], *[s if s is None else [s] for s in scales], copies=[c])
    opt.step(step=1, **HYPER)
    assert torch.equal(p, want.params[0]) and torch.equal(m, want.m[0]) and torch.equal(v, want.v[0]) and torch.equal(c, p)
    for b in bufs:
        assert bool((b[:off] == 5).all()) and bool((b[off + n:] == 5).all())
    got = opt.states()
    assert all(torch.equal(a[0], b[0]) for a, b in zip(got, want.states()))


def test_scaled_gradients():
    P, G = _make([3000], torch.float32, torch.float32, 6)
    a, b = [P[0].clone()], [P[0].clone()]
    ax.AxAdamW(a, G).step(step=1, grad_scale=torch.tensor([0.25], device="cuda"), **HYPER)
    ax.AxAdamW(b, [G[0] * 0.25]).step(step=1, **HYPER)
    assert torch.equal(a[0], b[0])


@pytest.mark.parametrize("bits", [32, 8])
def test_non_finite_gradients_show(bits):
    P, G = _make([1000], torch.float32, torch.float32, 7)
    G[0][300] = float("nan")
    opt = ax.AxAdamW(P, G, bits=bits)
    opt.step(step=1, **HYPER)
    bad = ~torch.isfinite(P[0].cpu())
    assert int(bad.sum()) == 1 and bool(bad[300])
    opt.step(step=2, **HYPER)
    bad = ~torch.isfinite(P[0].cpu())
    want = torch.zeros(1000, dtype=torch.bool)
    want[256:512] = True  # 8 bits: the block has lost its scale
    assert torch.equal(bad, want) if bits == 8 else int(bad.sum()) == 1


def test_states_of_small_values_in_8_bits():
    """Blocks of zeros, of values whose reciprocal leaves float32, and a second moment far below its block's largest."""
    P, G = _make([768], torch.float32, torch.float32, 8)
    G[0][:256] = 0
    G[0][256:512] = 1e-25  # squared: below what float32 holds
    G[0][512:] = 1e-6
    G[0][512] = 1.0
    opt = ax.AxAdamW(P, G, bits=8)
    opt.step(step=1, **HYPER)
    m, v = (t[0].cpu() for t in opt.states())
    assert not bool(m[:256].any()) and not bool(v[:512].any()) and bool((v[513:] > 0).all()) and bool((m[256:512] > 0).all())
    assert torch.isfinite(P[0]).all()


def test_more_elements_than_32_bits_count():
    n = (1 << 31) + 5000
    p, g = torch.zeros(n, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    tail = F.randn(F.gen(1), (4000,), 0.1, torch.bfloat16).cuda()
    p[-4000:], g[-4000:] = tail, tail
    opt = ax.AxAdamW([p], [g], bits=8)
    opt.step(step=1, **HYPER)
    q = torch.zeros(5000, dtype=torch.bfloat16, device="cuda")
    q[-4000:] = tail
    ref = ax.AxAdamW([q], [q.clone()], bits=8)
    ref.step(step=1, **HYPER)
    assert torch.equal(p[-5000:], q) and torch.equal(opt.m[0][-5000:], ref.m[0]) and torch.equal(opt.v[0][-5000:], ref.v[0])
    assert not bool(p[:-5000].any())
