"""CPU: more of what the layers of test_language_model_cpu.py do around the kernels."""
import copy
import pickle
import types

import pytest
import torch

from paper_2606_05613_gb300 import native
from paper_2606_05613_gb300.language import QueryKeyNorm, token_log_probs
from test_language_model_cpu import ROWS, _embedding, _gen, _places, _plain, _qk      # noqa: F401 (a fixture)


def test_a_layers_frequencies_are_its_own():
    """What a layer hands out cannot be written into another layer, or into a pass whose
    backward is still to come."""
    a, fused, q, k, pos = _qk()
    b = QueryKeyNorm(32, rotated=16, device="cpu")
    want = [10000.0 ** (-i / 8) for i in range(8)]
    qo, ko = a(q, k, pos)
    (ref,) = torch.autograd.grad((qo.float().sum() + ko.float().sum()), fused, retain_graph=True)
    with pytest.raises(TypeError):
        a.inv_freq[3] = 9.0
    assert list(a.inv_freq) == want and list(b.inv_freq) == want
    (again,) = torch.autograd.grad((qo.float().sum() + ko.float().sum()), fused)
    assert torch.equal(again, ref)


def test_a_layer_takes_frequencies():
    base, fused, q, k, pos = _qk()
    slow = [f / 4 for f in base.inv_freq]
    layer = QueryKeyNorm(32, device="cpu", inv_freq=slow)
    layer.load_state_dict(base.state_dict())
    slow[0] = 7.0                                 # (the caller's list stays the caller's)
    assert layer.rotated == 16 and layer.inv_freq == tuple(f / 4 for f in base.inv_freq)
    # a quarter of the frequency is the same turn at four times the position
    got, want = layer(q, k, 4 * pos), base(q, k, pos)
    assert all(torch.equal(u, v) for u, v in zip(got, want))
    for other in (pickle.loads(pickle.dumps(layer)), copy.deepcopy(layer)):
        assert other.inv_freq == layer.inv_freq
    for bad in (dict(rotated=32), dict(rotated=15)):
        with pytest.raises(ValueError, match="inv_freq"):
            QueryKeyNorm(32, device="cpu", inv_freq=layer.inv_freq, **bad)


@pytest.mark.parametrize("rotated", [17, 33, 8, 24, -16, 48])
def test_widths_that_cannot_be_rotated_are_refused(rotated):
    """17 elements were turned as 16 of them, by the frequencies of 17."""
    with pytest.raises(ValueError, match="rotated must be"):
        QueryKeyNorm(32, rotated=rotated, device="cpu")
    layer, _, q, k, pos = _qk()
    if rotated % 2:
        with pytest.raises(ValueError, match="even"):
            native.rope_frequencies(rotated, 1e4)
        layer.rotated = rotated                   # (an attribute that may be set)
        with pytest.raises(ValueError, match="even"):
            layer(q, k, pos)
    assert len(native.rope_frequencies(0, 1e4)) == 0 and QueryKeyNorm(32, rotated=0, device="cpu").inv_freq == ()


@pytest.mark.parametrize("apart", [True, False])
def test_one_weight_for_both_norms(monkeypatch, apart):
    """Queries' and keys' gradients of it add up; the call itself takes no places that overlap."""
    real = native.bkmoo_qk_norm_backward

    def strict(*a, **k):
        places = [*(a[11] or ()), *(a[12] or ())]
        assert len({p.data_ptr() for p in places}) == len(places)
        return real(*a, **k)

    monkeypatch.setattr(native, "bkmoo_qk_norm_backward", strict)
    layer, fused, q, k, pos = _qk()
    apart_layer, fused2, q2, k2, _ = _qk()
    layer.w_k = layer.w_q
    with torch.no_grad():
        apart_layer.w_k.copy_(apart_layer.w_q)
    if apart:
        for w in (layer.w_q, apart_layer.w_q, apart_layer.w_k):
            _places(w)
    for m, a, b in ((layer, q, k), (apart_layer, q2, k2)):
        qo, ko = m(a, b, pos, ROWS)
        (qo.float().square().sum() + ko.float().square().sum()).backward()
    assert torch.equal(fused.grad, fused2.grad)
    got = layer.w_q.language_grads if apart else [layer.w_q.grad]
    each = zip(apart_layer.w_q.language_grads, apart_layer.w_k.language_grads) if apart else [(apart_layer.w_q.grad, apart_layer.w_k.grad)]
    for g, (u, v) in zip(got, each):
        # each part is rounded to bf16, and their sum
        assert float((g.double() - (u.double() + v.double())).norm()) <= 2.0 ** -8 * float(u.double().norm() + v.double().norm() + g.double().norm())


@pytest.mark.parametrize("private", [True, False])
def test_workspaces_from_the_allocators_public_entries(monkeypatch, private):
    """The quicker entries that torch does not document are taken where they are there."""
    notes, names = [], ["_cuda_cudaCachingAllocator_raw_alloc", "_cuda_cudaCachingAllocator_raw_delete"]
    for name in names:
        monkeypatch.setattr(torch._C, name, None, raising=False)
        monkeypatch.delattr(torch._C, name)
    if private:
        monkeypatch.setattr(torch._C, names[0], lambda size, stream: notes.append((size, stream)) or 512, raising=False)
        monkeypatch.setattr(torch._C, names[1], lambda at: notes.append(at), raising=False)
    else:
        monkeypatch.setattr(torch.cuda, "caching_allocator_alloc",
                            lambda size, device=None, stream=None: notes.append((size, stream)) or (512 if device == 0 else 0))
        monkeypatch.setattr(torch.cuda, "caching_allocator_delete", lambda at: notes.append(at))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    stream = types.SimpleNamespace(cuda_stream=7)
    room = native._Room(torch, 100, 0, stream)
    assert room.at == 512
    del room
    native._Room(torch, 0, 0, stream)
    assert notes == [(100, 7), 512]


@pytest.mark.parametrize("lead", [(2, 5), (10,), (0, 5)])
def test_results_may_be_changed_in_place(lead):
    """x = embedding(ids); x += positions, and the like: the gradients are those of x = x + positions."""
    got = []
    for place in (True, False):
        emb, ids = _embedding(scale=2.0)
        x = emb(ids.reshape(-1)[:torch.Size(lead).numel()].view(lead))
        d = torch.randn(x.shape, generator=_gen(1)).bfloat16()
        x = x.add_(d) if place else x + d
        (x.float() ** 2).sum().backward()
        norm, fused, q, k, pos = _qk()
        q, k, pos = (t.flatten(0, 1)[:torch.Size(lead).numel()].view(*lead, *t.shape[2:]) for t in (q, k, pos))
        a, b = norm(q, k, pos)
        a, b = (a.mul_(0.5), b.add_(1.0)) if place else (a * 0.5, b + 1.0)
        ((a.float() ** 2).sum() + (b.float() ** 2).sum()).backward()
        z = torch.randn(*lead, 13, generator=_gen(2)).requires_grad_()
        t = torch.randint(0, 13, lead, generator=_gen(3))
        out = token_log_probs(z, t, entropy=True, top=2)
        skip = t < 4
        lp = out.logp.masked_fill_(skip, 0.0) if place else out.logp.masked_fill(skip, 0.0)
        assert lp.shape == out.entropy.shape == lead and out.top_ids.shape == (*lead, 2)
        ((lp ** 2).sum() + out.entropy.sum()).backward()
        got.append([x, emb.weight.grad, a, b, fused.grad, norm.w_q.grad, norm.w_k.grad, lp, z.grad])
    assert all(torch.equal(u, v) for u, v in zip(*got))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float64])
def test_log_probs_are_32_bit_under_any_default(dtype):
    z = torch.randn(5, 13, generator=_gen(2)).requires_grad_()
    t = torch.randint(0, 13, (5,), generator=_gen(3))
    torch.set_default_dtype(dtype)
    try:
        out = token_log_probs(z, t, entropy=True, top=2)
        assert all(v.dtype is torch.float32 for v in (out.logp, out.entropy, out.top_logp))
        out.entropy.sum().backward()
    finally:
        torch.set_default_dtype(torch.float32)
    assert z.grad.dtype is torch.float32
