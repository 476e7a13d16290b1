"""Layers whose weight gradients come apart by language, the optimizer on the
resolved direction, and the example that runs them together, on the GPU."""
import importlib.util
import os

import pytest
import torch

from paper_2606_05613_gb300 import native as bk
from paper_2606_05613_gb300.hook import BucketMOO
from paper_2606_05613_gb300.language import GatedFeedForward, LanguageLinear
from paper_2606_05613_gb300.optim import AdamW

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROWS = [0, 37, 37, 150]
K = 3


def _model(seed=0):
    torch.manual_seed(seed)
    return torch.nn.ModuleList([GatedFeedForward(72, 200, "silu"), LanguageLinear(72, 33)]).to(DEV)


def _plain(model, x):
    """The same by elementary operations, in 64 bits."""
    g, u, d, w = (p.double() for p in (model[0].w_gate, model[0].w_up, model[0].down.weight, model[1].weight))
    a = x.double() @ g.T
    return (a * torch.sigmoid(a) * (x.double() @ u.T)) @ d.T @ w.T


def _fused(model, x, rows):
    return model[1](model[0](x, rows), rows)


def _relative(a, b):
    return float((a.double() - b.double()).norm() / b.double().norm())


# bf16 results behind one another: 2^-9 each in the 2-norm (a rounding is at most 2^-9 of its value's
# binade, uniformly), at most eight of them on the way to a gradient (a, b, h, y, dy, dh, da or db, dW)
TOL = 8 * 2.0 ** -9


def test_gradients_come_apart_by_language():
    model = _model()
    params = list(model.parameters())
    moo = BucketMOO(params, K, 1 << 14, rule="mean")
    x = torch.randn(ROWS[-1], 72, device=DEV).bfloat16().requires_grad_()
    c = torch.randn(ROWS[-1], 33, device=DEV).bfloat16()
    moo.begin_batch()
    y = _fused(model, x, ROWS)
    y.backward(c)
    assert _relative(y, _plain(model, x)) <= TOL
    for k in range(K):
        i, j = ROWS[k], ROWS[k + 1]
        xk = x.detach()[i:j].clone().requires_grad_()
        ref = torch.autograd.grad((_plain(model, xk) * c[i:j].double()).sum(), params + [xk])
        for p, r in zip(params, ref):
            got = p.language_grads[k]
            if i == j:
                assert bool((got == 0).all())
            else:
                assert _relative(got, r) <= TOL
        if i < j:
            assert _relative(x.grad[i:j], ref[-1]) <= TOL
    grads = [g.clone() for g in moo.grads]
    d = moo.finish()
    # the direction is the resolve of those gradients, bit for bit
    out = torch.empty_like(d)
    bk.Resolver(K, torch.bfloat16, moo.layout.offsets, DEV).resolve(grads, "mean", out)
    assert torch.equal(d, out)
    assert all(p.grad is not None and p.language_grads is None for p in params)


def test_two_uses_of_a_weight_and_two_backward_passes_add_up():
    model = _model()
    moo = BucketMOO(model.parameters(), K, 1 << 14)
    x = torch.randn(ROWS[-1], 72, device=DEV).bfloat16()
    c = torch.randn(ROWS[-1], 33, device=DEV).bfloat16()
    moo.begin_batch()
    _fused(model, x, ROWS).backward(c)
    once = [g.clone() for g in moo.grads]
    moo.begin_batch()
    _fused(model, x, ROWS).backward(c)
    _fused(model, x, ROWS).backward(c)
    for a, b in zip(once, moo.grads):
        assert torch.equal(a * 2, b)          # a power of two: exact in bf16
    moo.finish()


def test_without_languages_the_ordinary_gradient():
    model = _model()
    params = list(model.parameters())
    x = torch.randn(50, 72, device=DEV).bfloat16()
    c = torch.randn(50, 33, device=DEV).bfloat16()
    _fused(model, x, None).backward(c)
    ref = torch.autograd.grad((_plain(model, x) * c.double()).sum(), params)
    for p, r in zip(params, ref):
        assert _relative(p.grad, r) <= TOL


def test_a_gradient_that_is_not_apart_is_refused():
    model = _model()
    moo = BucketMOO(model.parameters(), K, 1 << 14)
    moo.begin_batch()
    model[1].weight.float().sum().backward()
    with pytest.raises(RuntimeError):
        moo.finish()


def test_k_passes_still_work_after_a_batch():
    model = _model()
    params = list(model.parameters())
    moo = BucketMOO(params, K, 1 << 14, rule="mean")
    x = torch.randn(ROWS[-1], 72, device=DEV).bfloat16()
    c = torch.randn(ROWS[-1], 33, device=DEV).bfloat16()
    moo.begin_batch()
    _fused(model, x, ROWS).backward(c)
    batch = [g.clone() for g in moo.grads]
    moo.finish()
    for k in range(K):
        moo.begin(k)
        i, j = ROWS[k], ROWS[k + 1]
        if i < j:
            _fused(model, x[i:j], None).backward(c[i:j])
    for a, b in zip(batch, moo.grads):
        if float(b.float().norm()) > 0:
            assert _relative(a, b) <= TOL
    moo.finish()


@pytest.mark.parametrize("state", ["f32", "e4m3"])
@pytest.mark.parametrize("dtype,master", [(torch.float32, False), (torch.bfloat16, True), (torch.bfloat16, False)])
def test_optimizer_follows_torch(dtype, master, state):
    """Ten steps beside torch.optim.AdamW in fp32 (its own rounding is 2^-24 a step), with its clipping.
    8-bit moments are off by up to 1/16 each step: the step's direction must agree, not its bits."""
    torch.manual_seed(1)
    params = [torch.nn.Parameter(torch.randn(n, device=DEV).to(dtype)) for n in (1000, 3, 4097)]
    ref = [torch.nn.Parameter(p.detach().float().clone()) for p in params]
    decay = [0.1, 0.0, 0.1]
    opt = AdamW(params, lr=1e-2, betas=(0.9, 0.95), weight_decay=decay, max_norm=0.5, state=state, master=master)
    topt = torch.optim.AdamW([{"params": [p], "weight_decay": w} for p, w in zip(ref, decay)], lr=1e-2, betas=(0.9, 0.95))
    start = [p.detach().float().clone() for p in params]
    for _ in range(10):
        g = [torch.randn(p.shape, device=DEV) * 0.1 + 0.05 for p in params]
        for p, x in zip(ref, g):
            p.grad = x.clone()
        torch.nn.utils.clip_grad_norm_(ref, 0.5)
        topt.step()
        opt.step(torch.cat([x for x in reversed(g)]))
    for p, r, s in zip(params, ref, start):
        moved, want = p.detach().float() - s, r.detach() - s
        if state == "f32" and (master or dtype == torch.float32):
            half = 2.0 ** -8 if dtype == torch.bfloat16 else 0.0
            assert bool(((p.detach().float() - r).abs() <= half * r.abs() + 1e-5).all())
        elif r.numel() > 100 and (dtype == torch.float32 or master):
            assert float((moved * want).sum() / moved.norm() / want.norm()) > 0.9
    # the state carries over
    other = AdamW(params, lr=1e-2, betas=(0.9, 0.95), weight_decay=decay, max_norm=0.5, state=state, master=master)
    other.load_state_dict(opt.state_dict())
    d = torch.randn(5100, device=DEV)
    before = [p.detach().clone() for p in params]
    opt.step(d)
    after = [p.detach().clone() for p in params]
    with torch.no_grad():
        for p, b in zip(params, before):
            p.copy_(b)
    other.step(d)
    assert all(torch.equal(p, a) for p, a in zip(params, after))


def test_optimizer_refusals():
    p = [torch.nn.Parameter(torch.randn(8, device=DEV))]
    with pytest.raises(ValueError):
        AdamW(p, state="f16")
    with pytest.raises(ValueError):
        AdamW(p, master=True)
    with pytest.raises(ValueError):
        AdamW(p, weight_decay=[0.1, 0.2])
    with pytest.raises(ValueError):
        AdamW(p).load_state_dict(AdamW(p, state="e4m3").state_dict())
    with pytest.raises(ValueError):
        AdamW(p).step(torch.randn(9, device=DEV))


@pytest.mark.parametrize("rule", ["mgda", "cagrad"])
def test_example(rule):
    """The steps learn: every language's loss falls."""
    spec = importlib.util.spec_from_file_location("multilingual_step", os.path.join(ROOT, "examples", "multilingual_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    losses = m.run(steps=40, K=3, rule=rule)
    assert bool(torch.isfinite(losses).all())
    assert bool((losses[-1] < 0.8 * losses[0]).all()), losses[[0, -1]]
