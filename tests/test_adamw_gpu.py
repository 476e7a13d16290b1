"""AdamW over many tensors and the norm it clips by, on the GPU, against the
formulas in 64 bits.

Tolerances.  Moments of 32 bits: three roundings of 2^-24 of each term's
magnitude, and two more where the gradient is clipped (the factor and the
product); the second moment doubles the gradient's.  Weights: the old weight,
its decay and the difference are rounded once each, the step's quotient is good
to 2^-20 of it; bf16 weights add half an ulp, 2^-8.  Moments of 8 bits: a byte
must be the one that the formula gives in 64 bits, or its neighbour where the
threshold is nearer than fp32 can tell (16 steps a binade, a few roundings:
2^-17 of a step).
"""
import math

import numpy as np
import pytest
import torch

from paper_2606_05613_gb300 import native as bk

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
GOLD, M64 = 0x9E3779B97F4A7C15, (1 << 64) - 1
E = 2.0 ** -24


def _mix(z):
    z = ((z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9))
    z = ((z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB))
    return z ^ (z >> np.uint64(31))


def _chances(n, seed, step):
    with np.errstate(over="ignore"):
        key = _mix(np.array([(seed + (step + 1) * GOLD) & M64], dtype=np.uint64))
        z = _mix(key + np.arange(1, (n + 1) // 2 + 1, dtype=np.uint64) * np.uint64(GOLD))
    half = np.stack([z & np.uint64(0xFFFFFFFF), z >> np.uint64(32)], 1).reshape(-1)[:n]
    return [torch.tensor((h / 65536.0).astype(np.float64), device=DEV)
            for h in ((half & np.uint64(0xFFFF)), half >> np.uint64(16))]


def _per(scale, n):
    return scale.double().repeat_interleave(256)[:n]


def _e4m3(x):
    y = torch.nn.functional.pad(x, (0, -x.numel() % 256)).view(-1, 256)
    s = y.abs().amax(1) / 448
    return (y / s.clamp_min(1e-30)[:, None]).to(torch.float8_e4m3fn).view(-1)[:x.numel()].clone(), s


def _check_codes(code, scale, x, u, positive, what):
    """Bytes against the value in 64 bits, the scale as stored."""
    n = x.numel()
    pad = torch.nn.functional.pad(x.abs(), (0, -n % 256)).view(-1, 256).amax(1)
    pad = torch.where(pad < 2.0 ** -100, 0.0, pad)
    assert bool(((scale.double() - pad / 448).abs() <= 8 * E * pad / 448).all()), what
    y = torch.where(_per(scale, n) > 0, x.abs() / (pad.repeat_interleave(256)[:n] / 448).clamp_min(1e-300), 0.0)
    q = torch.exp2(torch.floor(torch.log2(y.clamp_min(2.0 ** -6))) - 3)
    t = y / q + u
    got = code.double()
    low, high = torch.floor(t - 2.0 ** -17) * q, torch.floor(t + 2.0 ** -17) * q
    if positive:
        least = torch.where(y > 0, 2.0 ** -9, 0.0)
        low, high = torch.maximum(low, least), torch.maximum(high, least)
    low, high = low.clamp(0, 448), high.clamp(0, 448)
    ok = (got.abs() == low) | (got.abs() == high)
    ok &= (got == 0) | (torch.sign(got) == torch.sign(x))
    assert bool(ok.all()), (what, int((~ok).sum()), [int(i) for i in (~ok).nonzero()[0]])


def _tensors(sizes, dtype, gen, how):
    """The weights: tensors of their own, or views at odd places of a framed buffer."""
    if how == "own":
        return [(torch.randn(n, generator=gen, device=DEV) * 0.02).to(dtype) for n in sizes], None
    n = sum(sizes) + 5 * len(sizes) + 8
    whole = torch.full((n,), 9.0, dtype=dtype, device=DEV)
    out, at = [], 1
    for k in sizes:
        out.append(whole[at:at + k])
        whole[at:at + k] = (torch.randn(k, generator=gen, device=DEV) * 0.02).to(dtype)
        at += k + 3
    return out, whole


def _flat(ts):
    return torch.cat([t.reshape(-1) for t in ts])


def _step(sizes, pd, gd, state, master, clip, how="own", decay="some", step=7, beta2=0.95, seed=3, steps=1):
    gen = torch.Generator(device=DEV).manual_seed(sum(sizes) + len(sizes))
    N = sum(sizes)
    ts, whole = _tensors(sizes, pd, gen, how)
    wd = [0.1 * (i % 3) for i in range(len(sizes))] if decay == "some" else None
    mast = _flat(ts).float() + 1e-5 * torch.randn(N, generator=gen, device=DEV) if master else None
    scale = torch.exp(torch.randn((N + 63) // 64, generator=gen, device=DEV)).repeat_interleave(64)[:N] * 1e-3
    scale[N // 3:N // 2] = 0.0                                # never touched
    m, r = torch.randn(N, generator=gen, device=DEV) * scale, (torch.rand(N, generator=gen, device=DEV) + 0.5) * scale
    ms = vs = None
    if state == "e4m3":
        (m, ms), (v, vs) = _e4m3(m), _e4m3(r)
    else:
        v = r * r
    p = bk.bkmoo_adamw_default_params()
    p.lr, p.beta2, p.seed = 3e-3, beta2, seed
    for k in range(steps):
        p.step = step + k
        g = (torch.randn(N, generator=gen, device=DEV) * scale).to(gd)
        old = [t.clone() for t in (_flat(ts).float() if mast is None else mast, m, v)]
        olds = [t.clone() for t in (ms, vs)] if state == "e4m3" else None
        norm = None
        if clip:
            norm = torch.empty(1, device=DEV)
            bk.bkmoo_grad_norm(g, norm)
            exact = torch.linalg.vector_norm(g.double())
            assert abs(float(norm) - float(exact)) <= 40 * E * float(exact)
            p.max_norm = float(exact) * 0.4
        bk.bkmoo_adamw(ts, g, m, v, params=p, weight_decay=wd, master=mast, m_scale=ms, v_scale=vs, grad_norm=norm)

        g = g.double()
        rel = 3
        if clip:
            g = g * min(1.0, p.max_norm / (float(norm) + 1e-6))
            rel = 6
        om, ov = old[1].double(), old[2].double()
        if olds:
            om, ov = om * _per(olds[0], N), (ov * _per(olds[1], N)) ** 2
        m64 = p.beta1 * om + (1 - p.beta1) * g
        v64 = p.beta2 * ov + (1 - p.beta2) * g * g
        em = rel * E * ((p.beta1 * om).abs() + ((1 - p.beta1) * g).abs())
        ev = 2 * rel * E * v64
        if olds:
            u = _chances(N, seed, p.step)
            _check_codes(m, ms, m64, u[0], False, "m")
            _check_codes(v, vs, v64.sqrt(), u[1], True, "v")
        else:
            assert bool(((m.double() - m64).abs() <= em + 1e-45).all())
            assert bool(((v.double() - v64).abs() <= ev + 1e-45).all())
        keep = 1 - p.lr * torch.tensor(wd or [0.0] * len(sizes), dtype=torch.float64, device=DEV).repeat_interleave(
            torch.tensor(sizes, device=DEV))
        den = (v64 / (1 - p.beta2 ** p.step)).sqrt() + p.eps
        up = p.lr / (1 - p.beta1 ** p.step) / den
        ref = old[0].double() * keep - up * m64
        err = 4 * E * (old[0].double().abs() + ref.abs()) + up * (em + m64.abs() * 2.0 ** -20)
        got = _flat(ts).double()
        if master:
            assert bool(((mast.double() - ref).abs() <= err).all())
            assert torch.equal(_flat(ts), mast.to(pd))
        else:
            half = 2.0 ** -8 if pd == torch.bfloat16 else 0.0
            assert bool(((got - ref).abs() <= err * 1.01 + half * ref.abs()).all())
    if whole is not None:
        mask = torch.ones_like(whole, dtype=torch.bool)
        at = 1
        for n in sizes:
            mask[at:at + n] = False
            at += n + 3
        assert bool((whole[mask] == 9).all())
    return ts, m, v, ms, vs


F, B = torch.float32, torch.bfloat16
TYPES = [(F, F, False), (F, B, False), (B, B, False), (B, F, False), (B, B, True), (B, F, True)]
SIZES = {"one": [1], "three": [3], "block": [256], "edge": [255, 2, 257], "tiny": [1] * 700 + [2, 0, 5] * 60,
         "ragged": [4097, 1, 0, 63, 20000, 129, 31, 70001, 5], "many": [37] * 2500,
         "empty ends": [0, 0, 300, 0], "multiples": [8192, 1024, 64, 4096]}


@pytest.mark.parametrize("state", ["f32", "e4m3"])
@pytest.mark.parametrize("sizes", list(SIZES))
@pytest.mark.parametrize("pd,gd,master", TYPES)
def test_step(pd, gd, master, sizes, state):
    for how in ("own", "views"):
        _step(SIZES[sizes], pd, gd, state, master, clip=len(SIZES[sizes]) > 2, how=how)


@pytest.mark.parametrize("state", ["f32", "e4m3"])
def test_several_steps_without_decay(state):
    _step([5000, 333], B, B, state, False, True, decay="none", step=1, beta2=0.999, steps=5)


@pytest.mark.parametrize("state", ["f32", "e4m3"])
def test_large(state):
    _step([20_000_003, 4_000_000], B, B, state, True, True)


def test_first_step_from_zeros():
    """The state before the first step is all zeros: the update is lr sign(g)."""
    N = 1000
    for dt in (torch.float32, torch.float8_e4m3fn):
        w = torch.zeros(N, device=DEV)
        g = torch.randn(N, device=DEV)
        g[100:400] = 0
        m, v = torch.zeros(N, device=DEV).to(dt), torch.zeros(N, device=DEV).to(dt)
        s = [torch.zeros(4, device=DEV) for _ in range(2)] if dt != torch.float32 else [None, None]
        p = bk.bkmoo_adamw_default_params()
        bk.bkmoo_adamw([w], g, m, v, params=p, m_scale=s[0], v_scale=s[1])
        # |m^| = |g|, sqrt(v^) + eps = |g| + 1e-8: quotients to 2^-20
        ref = -p.lr * g.double() / (g.double().abs() + p.eps)
        assert bool(((w.double() - ref).abs() <= 2.0 ** -19 * p.lr).all())
        assert bool((w[100:400] == 0).all()) and bool((m[100:400].float() == 0).all())


def test_roots_do_not_become_zero():
    """Small second moments beside a large one: bytes of at least 1."""
    N = 512
    g = torch.full((N,), 1e-9, device=DEV)
    g[0] = g[256] = 1.0
    m, v = (torch.zeros(N, device=DEV).to(torch.float8_e4m3fn) for _ in range(2))
    s = [torch.zeros(2, device=DEV) for _ in range(2)]
    w = torch.zeros(N, device=DEV)
    bk.bkmoo_adamw([w], g, m, v, m_scale=s[0], v_scale=s[1])
    assert bool((v.view(torch.uint8) >= 1).all())


def test_rounding_is_unbiased():
    """The mean of many rounded moments of one value is that value: 2^17 elements, a step of at most 1/8 of the
    value, so the mean's deviation is at most 1/16 / sqrt(2^17) of it; six of them."""
    N = 1 << 17
    g = torch.full((N,), 0.7, device=DEV)
    g[::256] = 1.0
    m, v = (torch.zeros(N, device=DEV).to(torch.float8_e4m3fn) for _ in range(2))
    s = [torch.zeros(N // 256, device=DEV) for _ in range(2)]
    p = bk.bkmoo_adamw_default_params()
    bk.bkmoo_adamw([torch.zeros(N, device=DEV)], g, m, v, params=p, m_scale=s[0], v_scale=s[1])
    keep = torch.arange(N, device=DEV) % 256 != 0
    for code, scale, ref in ((m, s[0], 0.1 * 0.7), (v, s[1], math.sqrt(0.001) * 0.7)):
        mean = float((code.double() * _per(scale, N))[keep].mean())
        assert abs(mean - ref) <= 6 * ref / 16 / math.sqrt(N)


def test_a_norm_that_is_not_finite_skips_the_step():
    for bad in (float("nan"), float("inf")):
        g = torch.randn(5000, device=DEV)
        g[4321] = bad
        norm = torch.empty((), device=DEV)
        bk.bkmoo_grad_norm(g, norm)
        assert not math.isfinite(float(norm))
        w, m, v = torch.randn(5000, device=DEV), torch.randn(5000, device=DEV), torch.rand(5000, device=DEV)
        old = [t.clone() for t in (w, m, v)]
        p = bk.bkmoo_adamw_default_params()
        for p.max_norm in (0.0, 1.0):
            bk.bkmoo_adamw([w], g, m, v, params=p, grad_norm=norm)
            assert all(torch.equal(a, b) for a, b in zip(old, (w, m, v)))
        p.max_norm = 0.0
        bk.bkmoo_adamw([w], g, m, v, params=p)
        assert not math.isfinite(float(w[4321])) and bool(torch.isfinite(w[:4000]).all())
        m8, v8 = (torch.zeros(5000, device=DEV).to(torch.float8_e4m3fn) for _ in range(2))
        s = [torch.zeros(20, device=DEV) for _ in range(2)]
        bk.bkmoo_adamw([w], g, m8, v8, params=p, m_scale=s[0], v_scale=s[1])
        assert not math.isfinite(float(m8[4321].float() * s[0][16]))


@pytest.mark.parametrize("dtype", [F, B])
@pytest.mark.parametrize("n", [0, 1, 3, 7, 8, 255, 16384, 16385, 3_000_001])
def test_norm(n, dtype):
    g = torch.randn(n, device=DEV).to(dtype)
    ws = torch.empty(bk.BKMOO_NORM_WS_BYTES, dtype=torch.uint8, device=DEV)
    a, b = torch.empty(1, device=DEV), torch.empty((), device=DEV)
    bk.bkmoo_grad_norm(g, a, ws=ws)
    bk.bkmoo_grad_norm(g, b)
    ref = float(torch.linalg.vector_norm(g.double())) if n else 0.0
    assert abs(float(a) - ref) <= 40 * E * ref
    assert float(a) == float(b)


def test_same_bits_on_streams_and_in_a_graph():
    sizes = [5001, 40_000, 77]
    N = sum(sizes)
    g = torch.randn(N, device=DEV)

    def make():
        w = [torch.ones(n, dtype=B, device=DEV) for n in sizes]
        m, v = (torch.zeros(N, device=DEV).to(torch.float8_e4m3fn) for _ in range(2))
        return w, m, v, [torch.zeros((N + 255) // 256, device=DEV) for _ in range(2)], torch.empty(1, device=DEV), \
            torch.empty(bk.BKMOO_NORM_WS_BYTES, dtype=torch.uint8, device=DEV)

    p = bk.bkmoo_adamw_default_params()
    p.max_norm = 1.0

    def go(o, stream=None):
        w, m, v, s, norm, ws = o
        bk.bkmoo_grad_norm(g, norm, ws=ws, stream=stream)
        bk.bkmoo_adamw(w, g, m, v, params=p, m_scale=s[0], v_scale=s[1], grad_norm=norm, stream=stream)

    outs = [make() for _ in range(4)]
    torch.cuda.synchronize()
    go(outs[0])
    for o in outs[1:3]:
        go(o, torch.cuda.Stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go(outs[3])
    graph.replay()
    torch.cuda.synchronize()
    for o in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(o[0], outs[0][0]))
        assert torch.equal(o[1].view(torch.uint8), outs[0][1].view(torch.uint8))
        assert torch.equal(o[2].view(torch.uint8), outs[0][2].view(torch.uint8))
        assert all(torch.equal(a, b) for a, b in zip(o[3], outs[0][3]))
