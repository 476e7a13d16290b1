"""What follows when a wait of the gate and weight-gradient kernels gives up: a wait of
their kind for an arrival that nothing makes, 1 ms long (bkmoo_selftest_give_up)."""
import pytest
import torch

from paper_2606_05613_gb300 import native as bk
from paper_2606_05613_gb300.hook import BucketMOO
from paper_2606_05613_gb300.language import GatedFeedForward
from paper_2606_05613_gb300.optim import AdamW

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ROWS = [0, 20, 50]


@pytest.fixture(autouse=True)
def _clear():
    bk.bkmoo_op_status(DEV)
    yield
    bk.bkmoo_op_status(DEV)


def test_the_word_says_so_until_it_is_read():
    bk.bkmoo_selftest_give_up(DEV)
    here, there = torch.zeros(1, dtype=torch.int32).pin_memory(), torch.zeros(1, dtype=torch.int32, device=DEV)
    for _ in range(2):                     # a copy does not clear it
        bk.bkmoo_op_status_copy(here)
        bk.bkmoo_op_status_copy(there)
        torch.cuda.synchronize()
        assert int(here) == int(there) == bk.BKMOO_ERR_TIMEOUT
    assert bk.bkmoo_op_status(DEV) == bk.BKMOO_ERR_TIMEOUT
    assert bk.bkmoo_op_status(DEV) == bk.BKMOO_OK
    for bad in (torch.zeros(1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32, device=DEV),
                torch.zeros(1, device=DEV)):
        with pytest.raises(ValueError):
            bk.bkmoo_op_status_copy(bad)


@pytest.mark.parametrize("max_norm", [0.0, 1.0])
@pytest.mark.parametrize("state", ["f32", "e4m3"])
def test_no_step_is_taken_with_undefined_gradients(state, max_norm):
    torch.manual_seed(0)
    params = [torch.nn.Parameter(torch.randn(n, device=DEV)) for n in (1000, 3, 4097)]
    opt = AdamW(params, lr=1e-2, max_norm=max_norm, state=state)
    d = torch.randn(5100, device=DEV)
    opt.step(d)

    def held():
        s = opt.state_dict()
        return [p.detach().clone() for p in params] + [t.view(torch.uint8).clone() if state == "e4m3" else t.clone()
                                                       for t in (s["m"], s["v"])]

    before = held()
    bk.bkmoo_selftest_give_up(DEV)
    opt.step(d)
    assert all(torch.equal(u, v) for u, v in zip(before, held()))
    assert bk.bkmoo_op_status(DEV) == bk.BKMOO_ERR_TIMEOUT
    opt.step(d)
    assert not any(torch.equal(u, v) for u, v in zip(before, held()))


def test_the_training_loop_hears_of_it():
    torch.manual_seed(0)
    layer = GatedFeedForward(64, 96).to(DEV)
    moo = BucketMOO(layer.parameters(), 2, 1 << 14, rule="mean")
    opt = AdamW(moo.params, lr=1e-2)
    x = torch.randn(ROWS[-1], 64, device=DEV).bfloat16()

    def step(give_up=False):
        moo.begin_batch()
        layer(x, ROWS).float().square().sum().backward()
        if give_up:
            bk.bkmoo_selftest_give_up(DEV)
        opt.step(moo.finish())

    step()
    torch.cuda.synchronize()
    before = [p.detach().clone() for p in moo.params]
    step(give_up=True)
    torch.cuda.synchronize()
    assert all(torch.equal(u, v) for u, v in zip(before, moo.params))
    with pytest.raises(bk.BkmooError) as e:
        moo.begin_batch()
    assert e.value.code == bk.BKMOO_ERR_TIMEOUT
    step()
    step()
    torch.cuda.synchronize()
    assert not any(torch.equal(u, v) for u, v in zip(before, moo.params))
    moo.begin_batch()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_norm_of_an_undefined_gradient(dtype):
    g, norm = torch.ones(1 << 16, dtype=dtype, device=DEV), torch.zeros((), device=DEV)
    bk.bkmoo_selftest_give_up(DEV)
    bk.bkmoo_grad_norm(g, norm)
    assert bool(torch.isnan(norm))
    assert bk.bkmoo_op_status(DEV) == bk.BKMOO_ERR_TIMEOUT
    bk.bkmoo_grad_norm(g, norm)
    assert float(norm) == 256.0


@pytest.mark.parametrize("ctas", [1, 2])
def test_a_kernel_without_its_operands_ends(ctas):
    """Each of its waits ends, it hands back its tensor memory and says so; what runs behind
    it, on every SM, is right."""
    torch.manual_seed(0)
    x, w = torch.randn(2051, 520, device=DEV).bfloat16(), (torch.randn(2 * 4104, 520, device=DEV) * 0.05).bfloat16()
    first, after = (torch.empty(2051, 4104, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    bk.bkmoo_gate_forward(x, w[:4104], w[4104:], "silu", first)
    for _ in range(2):
        bk.bkmoo_selftest_give_up(DEV, ctas)
    bk.bkmoo_gate_forward(x, w[:4104], w[4104:], "silu", after)
    assert bk.bkmoo_op_status(DEV) == bk.BKMOO_ERR_TIMEOUT
    assert torch.equal(first, after)
    bk.bkmoo_gate_forward(x, w[:4104], w[4104:], "silu", after)
    assert bk.bkmoo_op_status(DEV) == bk.BKMOO_OK
