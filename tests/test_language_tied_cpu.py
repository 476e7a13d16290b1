"""CPU: one parameter as both weights of the gated projections.  The kernels' outputs must not
overlap, so its places go to a call at a time."""
import pytest
import torch

from paper_2606_05613_gb300 import native
from paper_2606_05613_gb300.language import GatedFeedForward
from test_language_cpu import _built, _gate_backward, _input, _places, _plain      # noqa: F401 (fixtures)

ROWS = [0, 4, 4, 10]


@pytest.mark.parametrize("apart", [True, False])
def test_one_weight_for_gate_and_up(monkeypatch, apart):
    def strict(*a, **k):
        places = [p.data_ptr() for side in a[9:11] if side is not None for p in side]
        assert len(set(places)) == len(places)
        return _gate_backward(*a, **k)

    monkeypatch.setattr(native, "bkmoo_gate_backward", strict)
    torch.manual_seed(0)
    tied, both = GatedFeedForward(24, 40, device="cpu"), GatedFeedForward(24, 40, device="cpu")
    tied.w_up = tied.w_gate
    both.load_state_dict(tied.state_dict())
    if apart:
        for p in [*tied.parameters(), *both.parameters()]:
            _places(p)
    x, y = _input(), _input()
    for layer, z in ((tied, x), (both, y)):
        layer(z, ROWS).float().square().sum().backward()
    assert torch.equal(x.grad, y.grad)
    got = tied.w_gate.language_grads if apart else [tied.w_gate.grad]
    each = zip(both.w_gate.language_grads, both.w_up.language_grads) if apart else [(both.w_gate.grad, both.w_up.grad)]
    for g, (u, v) in zip(got, each):
        # each part is rounded to bf16, and their sum
        bound = 2.0 ** -8 * float(u.double().norm() + v.double().norm() + g.double().norm())
        assert float((g.double() - (u.double() + v.double())).norm()) <= bound
