"""CPU: what the layers of language.py do around the kernels, which plain products
stand in for here."""
import pytest
import torch

from paper_2606_05613_gb300 import build as nb
from paper_2606_05613_gb300 import native
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


@pytest.fixture(scope="module", autouse=True)
def _built():
    nb.build()


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


ROWS = [0, 4, 4, 10]


def _places(weight, K=3):
    weight.language_grads = [torch.zeros(weight.shape, dtype=torch.bfloat16) for _ in range(K)]
    return weight.language_grads


@pytest.mark.parametrize("input_grad", [True, False])
@pytest.mark.parametrize("apart", [True, False])
@pytest.mark.parametrize("frozen", ["w_gate", "w_up"])
def test_one_of_the_gated_weights_is_frozen(frozen, apart, input_grad):
    """The other one's gradients are what they are with both of them trained, apart by
    language or not, and nothing is computed for the frozen one."""
    def layer():
        torch.manual_seed(2)
        return GatedFeedForward(24, 40, device="cpu")

    got = []
    for freeze in (False, True):
        f = layer()
        if freeze:
            getattr(f, frozen).requires_grad_(False)
        trained = [p for p in f.parameters() if p.requires_grad]
        places = [_places(p) for p in trained] if apart else None
        x = _input().detach().requires_grad_(input_grad)
        f(x, ROWS).float().square().sum().backward()
        other = f.w_up if frozen == "w_gate" else f.w_gate
        got.append(([x.grad] if input_grad else []) + (other.language_grads if apart else [other.grad]))
        if freeze:
            assert getattr(f, frozen).grad is None
        if apart:
            assert all(p.grad is None for p in trained) and places is not None
    assert len(got[0]) == len(got[1]) and all(torch.equal(u, v) for u, v in zip(*got))


def test_one_of_the_gated_weights_is_not_apart():
    """A weight without places for its languages gets the ordinary gradient beside one that has."""
    torch.manual_seed(3)
    f = GatedFeedForward(24, 40, device="cpu")
    both = GatedFeedForward(24, 40, device="cpu")
    both.load_state_dict(f.state_dict())
    _places(f.w_up)
    f(_input(), ROWS).float().square().sum().backward()
    both(_input()).float().square().sum().backward()
    assert torch.equal(f.w_gate.grad, both.w_gate.grad) and f.w_up.grad is None
    total = sum(g.float() for g in f.w_up.language_grads)
    # the languages' sums rounded once each, against the whole batch's rounded once
    assert float((total - both.w_up.grad.float()).norm()) <= 2 * 2.0 ** -9 * float(both.w_up.grad.float().norm())


def test_bounds_must_fit_the_languages():
    f = GatedFeedForward(24, 40, device="cpu")
    _places(f.w_gate)
    _places(f.w_up)
    with pytest.raises(ValueError, match="bounds of the 3 languages"):
        f(_input(), [0, 4, 10]).float().sum().backward()


class _Stream:
    """A stream by name that notes what it waits for."""
    notes = []

    def __init__(self, name):
        self.cuda_stream = name

    def wait_stream(self, other):
        self.notes.append((self.cuda_stream, "waits for", other.cuda_stream))


@pytest.mark.parametrize("layer", ["gate", "linear"])
@pytest.mark.parametrize("current", ["home", "other"])
def test_gradients_written_on_another_stream(monkeypatch, layer, current):
    """What zeroed and what resolves the places is on the stream of begin_batch(); where a
    backward pass runs on another, each waits for the other around the write."""
    from paper_2606_05613_gb300.hook import LanguageGrads
    home, now = _Stream("home"), _Stream(current)
    monkeypatch.setattr(_Stream, "notes", [])
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: now)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: now.cuda_stream, raising=False)

    def noted(fn):
        def call(*a, **k):
            _Stream.notes.append("write")
            return fn(*a, **k)
        return call

    monkeypatch.setattr(native, "bkmoo_gate_backward", noted(_gate_backward))
    monkeypatch.setattr(native, "bkmoo_language_wgrad", noted(_language_wgrad))
    torch.manual_seed(0)
    f = GatedFeedForward(24, 40, device="cpu") if layer == "gate" else LanguageLinear(24, 40, device="cpu")
    for p in f.parameters():
        p.language_grads = LanguageGrads([torch.zeros(p.shape, dtype=torch.bfloat16) for _ in range(3)], home, 0)
    f(_input(), ROWS).float().square().sum().backward()
    one = ["write"] if current == "home" else [("other", "waits for", "home"), "write", ("home", "waits for", "other")]
    # (the gated call writes two weights' places, each of which takes care of itself)
    def once(notes):
        return [n for i, n in enumerate(notes) if i == 0 or n != notes[i - 1]]

    assert once(_Stream.notes) == once(one * (2 if layer == "gate" else 1))
