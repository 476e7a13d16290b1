"""The optimizer object on the GPU: parameters whose storage is replaced, refused steps,
its state."""
import pytest
import torch

from paper_2606_05613_gb300 import native as bk
from paper_2606_05613_gb300.optim import AdamW

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SIZES = (1000, 3, 4097)


def _params(dtype=torch.float32, seed=0):
    torch.manual_seed(seed)
    return [torch.nn.Parameter(torch.randn(n, device=DEV).to(dtype)) for n in SIZES]


def _direction(seed=1):
    return torch.randn(sum(SIZES), device=DEV, generator=torch.Generator(device=DEV).manual_seed(seed))


@pytest.mark.parametrize("dtype,master", [(torch.float32, False), (torch.bfloat16, True), (torch.bfloat16, False)])
def test_parameters_that_move_are_followed(dtype, master):
    """p.data = ... between two steps: the step goes to the new storage, as if nothing had moved."""
    ends = []
    for move in (False, True):
        params = _params(dtype)
        opt = AdamW(params, lr=1e-2, weight_decay=0.1, master=master)
        for i in range(3):
            if move:
                old = [p.data for p in params]
                for p in params:
                    p.data = p.data.clone()
                kept = [o.clone() for o in old]
            opt.step(_direction(i))
            if move:
                assert all(torch.equal(o, k) for o, k in zip(old, kept))      # nothing is written there
        ends.append([p.detach().clone() for p in params])
    assert all(torch.equal(u, v) for u, v in zip(*ends))


def test_parameters_that_change_are_refused():
    params = _params()
    opt = AdamW(params)
    d = _direction()
    opt.step(d)
    kept = params[2].data
    for other in (kept.bfloat16(), kept.cpu(), kept[:4000], kept.repeat(2)[::2]):
        params[2].data = other
        with pytest.raises(ValueError):
            opt.step(d)
    params[2].data = kept
    opt.step(d)


def test_a_tensor_list_follows_too():
    p = _params()
    tensors = bk.TensorList(p, 0.1)
    m, v = torch.zeros(sum(SIZES), device=DEV), torch.zeros(sum(SIZES), device=DEV)
    bk.bkmoo_adamw(tensors, _direction(), m, v)
    for t in p:
        t.data = torch.full_like(t.data, 2.0)
    bk.bkmoo_adamw(tensors, torch.zeros(sum(SIZES), device=DEV), torch.zeros_like(m), torch.zeros_like(v))
    for t in p:                            # only the decay is left of that step
        assert bool(((t.detach() - 2.0 * (1.0 - 1e-4)).abs() <= 2.0 ** -22).all())


@pytest.mark.parametrize("size", [1e-18, 1e-19, 3e-20])
def test_second_moments_below_the_normal_numbers(size):
    """Gradients whose squares fp32 holds as subnormal numbers only, and no eps: the first
    step is the rate, as the formula has it.  (1 - beta2) g^2 is a multiple of 2^-149, so its
    root is off by at most 2^-150 of it; the rest are fp32 roundings."""
    p = [torch.nn.Parameter(torch.zeros(n, device=DEV)) for n in SIZES]
    opt = AdamW(p, lr=1e-2, betas=(0.9, 0.95), eps=0.0)
    g = torch.where(_direction() > 0, size, -size)
    opt.step(g)
    off = 2.0 ** -150 / (0.05 * size * size) + 2.0 ** -150 / (size * size) + 2.0 ** -18
    flat = torch.cat([t.detach() for t in reversed(p)])
    assert bool(((flat + 1e-2 * torch.sign(g)).abs() <= 1e-2 * off).all())


@pytest.mark.parametrize("state", ["f32", "e4m3"])
def test_bf16_parameters_without_a_master_copy(state):
    """Every step against the formula in 64 bits from the weights and moments before it: the
    weights widened, stepped and rounded to nearest, 2^-8 of them at most, beside the fp32
    step's own roundings (the rate is 1e-2, a first moment over the root at most 10)."""
    p = _params(torch.bfloat16)
    lr, b1, b2, eps, decay = 1e-2, 0.9, 0.95, 1e-8, 0.1
    opt = AdamW(p, lr=lr, betas=(b1, b2), eps=eps, weight_decay=decay, max_norm=0.5, state=state)

    def flat():
        return torch.cat([t.detach() for t in reversed(p)]).double()

    def moment(code, scale):
        return code.double() if scale is None else code.double() * scale.double().repeat_interleave(256)[:code.numel()]

    for t in range(1, 11):
        g = _direction(t)
        w, m, v = flat(), moment(opt.m, opt.m_scale), moment(opt.v, opt.v_scale)
        opt.step(g)
        g = g.double() * min(1.0, 0.5 / (float(g.double().norm()) + 1e-6))
        m = b1 * m + (1 - b1) * g
        v = b2 * (v if state == "f32" else v * v) + (1 - b2) * g * g
        want = w * (1 - lr * decay) - lr * (m / (1 - b1 ** t)) / (torch.sqrt(v / (1 - b2 ** t)) + eps)
        assert bool(((flat() - want).abs() <= 2.0 ** -8 * want.abs() + 10 * lr * 2.0 ** -18).all())
