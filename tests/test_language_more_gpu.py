"""Layers of languages on the GPU: weights that are not all trained, passes on another
stream."""
import pytest
import torch

from paper_2606_05613_gb300.hook import BucketMOO
from paper_2606_05613_gb300.language import GatedFeedForward

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ROWS = [0, 37, 37, 150]
K = 3
# bf16 results behind one another: 2^-9 each in the 2-norm, at most eight of them on the way
# to a gradient
TOL = 8 * 2.0 ** -9


def _plain(layer, x):
    """The layer by elementary operations, in 64 bits."""
    g, u, d = (p.double() for p in (layer.w_gate, layer.w_up, layer.down.weight))
    a = x.double() @ g.T
    return (a * torch.sigmoid(a) * (x.double() @ u.T)) @ d.T


def _relative(a, b):
    return float((a.detach().double() - b).norm() / b.norm())


@pytest.mark.parametrize("input_grad", [True, False])
@pytest.mark.parametrize("frozen", ["w_gate", "w_up"])
def test_one_of_the_gated_weights_is_frozen(frozen, input_grad):
    torch.manual_seed(0)
    layer = GatedFeedForward(72, 201).to(DEV)
    getattr(layer, frozen).requires_grad_(False)
    trained = [p for p in layer.parameters() if p.requires_grad]
    moo = BucketMOO(layer.parameters(), K, 1 << 14, rule="mean")
    x = torch.randn(ROWS[-1], 72, device=DEV).bfloat16().requires_grad_(input_grad)
    c = torch.randn(ROWS[-1], 72, device=DEV).bfloat16()
    moo.begin_batch()
    layer(x, ROWS).backward(c)
    for k, (i, j) in enumerate(zip(ROWS, ROWS[1:])):
        xk = x.detach()[i:j].clone().requires_grad_()
        ref = torch.autograd.grad((_plain(layer, xk) * c[i:j].double()).sum(), trained + [xk])
        for p, r in zip(trained, ref):
            assert bool((p.language_grads[k] == 0).all()) if i == j else _relative(p.language_grads[k], r) <= TOL
        if input_grad and i < j:
            assert _relative(x.grad[i:j], ref[-1]) <= TOL
    moo.finish()
    assert getattr(layer, frozen).grad is None


class _Late(torch.autograd.Function):
    """Keeps the stream of its backward pass busy for some milliseconds first."""

    @staticmethod
    def forward(ctx, y):
        return y.clone()

    @staticmethod
    def backward(ctx, dy):
        torch.cuda._sleep(20_000_000)
        return dy.clone()


def test_a_pass_on_another_stream():
    """begin_batch() and finish() on one stream, the model's passes on another that is late:
    the direction is that of a run on one stream, bit for bit."""
    torch.manual_seed(1)
    layer = GatedFeedForward(72, 200).to(DEV)
    moo = BucketMOO(layer.parameters(), K, 1 << 14, rule="mean")
    x = torch.randn(ROWS[-1], 72, device=DEV).bfloat16()
    c = torch.randn(ROWS[-1], 72, device=DEV).bfloat16()
    other = torch.cuda.Stream()

    def run(stream):
        moo.begin_batch()
        if stream is None:
            layer(x, ROWS).backward(c)
        else:
            stream.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(stream):
                y = _Late.apply(layer(x, ROWS))
            y.backward(c)
        return moo.finish().clone(), [g.clone() for g in moo.grads]

    d, grads = run(None)
    for _ in range(2):
        late, late_grads = run(other)
        assert torch.equal(d, late) and all(torch.equal(u, v) for u, v in zip(grads, late_grads))
    torch.cuda.synchronize()
