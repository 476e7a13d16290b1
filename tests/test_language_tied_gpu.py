"""One parameter as both weights of a layer, in a batch of all languages, on the GPU."""
import pytest
import torch

from paper_2606_05613_gb300.hook import BucketMOO
from paper_2606_05613_gb300.language import GatedFeedForward, QueryKeyNorm

pytestmark = pytest.mark.gpu
ROWS = [0, 37, 37, 150]


def _run(layer, step):
    params = list(layer.parameters())
    moo = BucketMOO(params, 3, 1 << 14, rule="mean")
    moo.begin_batch()
    out = step(layer)
    grads = {n: [g.double().clone() for g in p.language_grads] for n, p in layer.named_parameters()}
    moo.finish()
    moo.remove()
    return out, grads


def _check(tied, both, step, names):
    x, got = _run(tied, step)
    y, each = _run(both, step)
    assert torch.equal(x, y)
    for g, u, v in zip(got[names[0]], each[names[0]], each[names[1]]):
        # each part is rounded to bf16, and their sum
        assert float((g - (u + v)).norm()) <= 2.0 ** -8 * float(u.norm() + v.norm() + g.norm())
    assert float(got[names[0]][0].norm()) > 0 and float(got[names[0]][1].norm()) == 0


def test_norms():
    gen = torch.Generator(device="cuda").manual_seed(1)
    q, k, cq, ck = (torch.randn(150, h, 64, generator=gen, device="cuda").bfloat16() for h in (6, 2, 6, 2))
    pos = torch.arange(150, device="cuda")

    def step(layer):
        a, b = q.clone().requires_grad_(), k.clone().requires_grad_()
        torch.autograd.backward(layer(a, b, pos, ROWS), (cq, ck))
        return torch.cat([a.grad, b.grad], 1)

    tied, both = QueryKeyNorm(64), QueryKeyNorm(64)
    tied.w_k = tied.w_q
    _check(tied, both, step, ("w_q", "w_k"))


def test_gated_projections():
    torch.manual_seed(2)
    x, c = (torch.randn(150, 72, device="cuda").bfloat16() for _ in range(2))

    def step(layer):
        a = x.clone().requires_grad_()
        layer(a, ROWS).backward(c)
        return a.grad

    tied, both = GatedFeedForward(72, 136), GatedFeedForward(72, 136)
    tied.w_up = tied.w_gate
    with torch.no_grad():
        for w, v in ((both.w_gate, tied.w_gate), (both.w_up, tied.w_gate), (both.down.weight, tied.down.weight)):
            w.copy_(v)
    _check(tied, both, step, ("w_gate", "w_up"))
