"""CPU: what the layers of language.py do around the kernels, which plain products
stand in for here."""
import pytest
import torch

from paper_2606_05613_gb300 import language, native
from paper_2606_05613_gb300.language import GatedFeedForward, LanguageLinear


def _act(a):
    s = torch.sigmoid(a)
    return a * s, s * (1 + a * (1 - s))


def _store(dw, value, accumulate):
    for place, v in zip(dw, value):
        place.copy_(place.float() + v if accumulate else v)


def _by_language(d, x, rows):
    return [d[i:j].T @ x[i:j] for i, j in zip(rows, rows[1:])]


def _gate_forward(x, w_gate, w_up, act, h=None, a=None, b=None, stream=None):
    p, q = x.float() @ w_gate.float().T, x.float() @ w_up.float().T
    if h is not None:
        h.copy_(_act(p)[0] * q)
    if a is not None:
        a.copy_(p)
        b.copy_(q)


def _gate_backward(dh, a, b, x, w_gate, w_up, act, rows, dx=None, dw_gate=None, dw_up=None, accumulate=False, ws=None,
                   stream=None):
    if (dw_gate is None) != (dw_up is None) or (dw_gate is not None and not len(dw_gate) == len(dw_up) == len(rows) - 1):
        raise ValueError("one gradient per language")
    T, F = a.shape
    f, df = _act(a.float())
    da, db = (dh.float() * b.float() * df).bfloat16(), (dh.float() * f).bfloat16()
    if ws is not None:                     # da and db, each from a multiple of 256 bytes on
        ld, half = (F + 7) // 8 * 8, ws.numel() // 2
        for i, d in enumerate((da, db)):
            ws[i * half:i * half + T * ld * 2].view(torch.bfloat16).view(T, ld)[:, :F].copy_(d)
    da, db, x = da.float(), db.float(), x.float()
    if dx is not None:
        dx.copy_(da @ w_gate.float() + db @ w_up.float())
    if dw_gate is not None:
        _store(dw_gate, _by_language(da, x, rows), accumulate)
        _store(dw_up, _by_language(db, x, rows), accumulate)


def _language_wgrad(dy, x, rows, dw, accumulate=False, stream=None):
    if len(dw) != len(rows) - 1:
        raise ValueError("one gradient per language")
    _store(dw, _by_language(dy.float(), x.float(), rows), accumulate)


@pytest.fixture(autouse=True)
def _plain(monkeypatch):
    monkeypatch.setattr(native, "bkmoo_gate_forward", _gate_forward)
    monkeypatch.setattr(native, "bkmoo_gate_backward", _gate_backward)
    monkeypatch.setattr(native, "bkmoo_language_wgrad", _language_wgrad)


def _input(T=10, D=24, seed=0):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(T, D, generator=g).bfloat16().requires_grad_()


@pytest.mark.parametrize("make", [lambda: GatedFeedForward(24, 40, device="cpu"), lambda: LanguageLinear(24, 16, device="cpu")])
def test_gradients_of_gradients_are_refused(make):
    """The kernels' results have no graph of their own: asking for a gradient of a gradient
    says so instead of leaving terms out."""
    torch.manual_seed(0)
    layer, x = make(), _input()
    y = layer(x * x)
    (g,) = torch.autograd.grad(y.float().square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        g.float().square().sum().backward()


def test_layers_give_the_gradients_of_the_formula():
    torch.manual_seed(1)
    layer, x = GatedFeedForward(24, 40, device="cpu"), _input()
    y = layer(x)
    params = [layer.w_gate, layer.w_up, layer.down.weight]
    got = torch.autograd.grad(y.float().square().sum(), params + [x])
    wide = [p.detach().double().requires_grad_() for p in params + [x]]
    p, q, d, z = wide
    ref = torch.autograd.grad((((_act(z @ p.T)[0] * (z @ q.T)) @ d.T).square()).sum(), wide)
    for g, r in zip(got, ref):
        # at most eight bf16 roundings behind one another, 2^-9 each in the 2-norm
        assert float((g.double() - r).norm() / r.norm()) <= 8 * 2.0 ** -9
