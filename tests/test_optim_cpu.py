"""CPU: the bookkeeping of the optimizer object, without its kernels."""
import pytest
import torch

from paper_2606_05613_gb300 import build as nb
from paper_2606_05613_gb300 import native
from paper_2606_05613_gb300.optim import AdamW


@pytest.fixture(scope="module", autouse=True)
def _built():
    nb.build()


class _Tensors:
    def __init__(self, tensors):
        self.tensors = tensors


def _optimizer(params=()):
    """An optimizer of CPU parameters, as its constructor leaves one of GPU parameters."""
    opt = AdamW.__new__(AdamW)
    opt.tensors = _Tensors(list(reversed(params)))
    opt.p = native.bkmoo_adamw_default_params()
    opt.p.step, opt.p.seed, opt.p.lr = 0, 77, 0.5
    opt.m, opt.v = torch.zeros(8), torch.zeros(8)
    opt.m_scale = opt.v_scale = opt.master = opt.norm = opt._ws = None
    return opt


def test_state_keeps_the_seed_of_the_rounding():
    """Resumed steps draw what the run itself would have drawn."""
    one, other = _optimizer(), _optimizer()
    one.p.step, other.p.seed = 12, 5
    other.load_state_dict(one.state_dict())
    assert (other.p.step, other.p.seed) == (12, 77)
    old = one.state_dict()
    del old["seed"]                        # a state that was saved without one
    other.p.seed = 5
    other.load_state_dict(old)
    assert (other.p.step, other.p.seed) == (12, 5)


def test_a_refused_step_does_not_count(monkeypatch):
    """The step's number goes into the bias corrections and the rounding: a call that is
    refused leaves it, and the rate, as they were."""
    opt = _optimizer()

    def refuse(*a, **k):
        raise ValueError("grad")

    monkeypatch.setattr(native, "bkmoo_adamw", refuse)
    with pytest.raises(ValueError):
        opt.step(torch.zeros(9), lr=2.0)
    assert (opt.p.step, opt.p.lr) == (0, 0.5)
    taken = []
    monkeypatch.setattr(native, "bkmoo_adamw", lambda *a, **k: taken.append((k["params"].step, k["params"].lr)))
    opt.step(torch.zeros(8))
    opt.step(torch.zeros(8), lr=2.0)
    opt.step(torch.zeros(8))
    assert taken == [(1, 0.5), (2, 2.0), (3, 2.0)] and opt.p.step == 3


def test_a_pass_that_spans_a_step_is_refused(monkeypatch):
    """Weights that a step has changed since the forward pass are not the ones its backward
    pass needs: autograd says so, as it does for torch's optimizers."""
    monkeypatch.setattr(native, "bkmoo_adamw", lambda *a, **k: None)
    w = torch.nn.Parameter(torch.randn(4, 4))
    opt = _optimizer([w])
    x = torch.randn(2, 4, requires_grad=True)
    (x @ w).sum().backward()
    opt.step(torch.zeros(16))
    y = x @ w
    opt.step(torch.zeros(16))
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
