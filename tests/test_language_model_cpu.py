"""CPU: what the embedding, the norms of queries and keys and the log probabilities of
language.py do around the kernels, which plain operations stand in for here."""
import math
import pickle

import pytest
import torch

from paper_2606_05613_gb300 import native
from paper_2606_05613_gb300.language import Embedding, LanguageLinear, QueryKeyNorm, token_log_probs

ROWS = [0, 4, 4, 10]
T, K = 10, 3


def _scale(ids, V, scale):
    return ((ids >= 0) & (ids < V)).float()[:, None] * scale


def _embedding_forward(table, ids, out, scale=1.0, stream=None):
    V = table.shape[0]
    out.copy_(table.float()[ids.long().clamp(0, V - 1)] * _scale(ids, V, scale))


def _embedding_backward(dy, ids, rows, dw, scale=1.0, accumulate=False, ws=None, stream=None):
    if len(dw) != len(rows) - 1:
        raise ValueError("one gradient per language")
    V = dw[0].shape[0]
    for w, i, j in zip(dw, rows, rows[1:]):
        g = torch.zeros(w.shape).index_add_(0, ids[i:j].long().clamp(0, V - 1), dy[i:j].float() * _scale(ids[i:j], V, scale))
        w.copy_(w.float() + g if accumulate else g)


def _normed(x, w, pos, freq, eps, interleaved):
    y = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) * w
    rot = 2 * len(freq)
    a = pos.double()[:, None] * torch.tensor(list(freq), dtype=torch.float64)
    c, s = (t.to(x.dtype)[:, None] for t in (a.cos(), a.sin()))
    u, v = (y[..., 0:rot:2], y[..., 1:rot:2]) if interleaved else (y[..., :rot // 2], y[..., rot // 2:rot])
    u, v = u * c - v * s, v * c + u * s
    z = torch.stack([u, v], -1).flatten(-2) if interleaved else torch.cat([u, v], -1)
    return torch.cat([z, y[..., rot:]], -1)


def _qk_forward(q, k, w_q, w_k, positions, inv_freq, q_out, k_out, eps=1e-6, interleaved=False, stream=None):
    for x, w, o in ((q, w_q, q_out), (k, w_k, k_out)):
        o.copy_(_normed(x.float(), w.float(), positions, inv_freq, eps, interleaved))


calls = []


def _qk_backward(dq_out, dk_out, q, k, w_q, w_k, positions, inv_freq, rows, dq, dk, dw_q=None, dw_k=None, eps=1e-6,
                 interleaved=False, accumulate=False, ws=None, stream=None):
    calls.append((dw_q is not None, dw_k is not None))
    if (dw_q is None) != (dw_k is None) or (dw_q is not None and not len(dw_q) == len(dw_k) == len(rows) - 1):
        raise ValueError("one gradient per language")
    for x, w, do, d, dw in ((q, w_q, dq_out, dq, dw_q), (k, w_k, dk_out, dk, dw_k)):
        for i, (a, b) in enumerate(zip(rows, rows[1:])):
            with torch.enable_grad():
                xs, ws_ = x[a:b].float().requires_grad_(), w.float().requires_grad_()
                y = _normed(xs, ws_, positions[a:b], inv_freq, eps, interleaved)
                gx, gw = torch.autograd.grad(y, (xs, ws_), do[a:b].float())
            d[a:b] = gx
            if dw is not None:
                dw[i].copy_(dw[i].float() + gw if accumulate else gw)


def _logp_forward(logits, targets, logp, stats=None, entropy=None, top_ids=None, top_logp=None, stream=None):
    z, V = logits.float(), logits.shape[1]
    lp = z.log_softmax(-1)
    ok = (targets >= 0) & (targets < V)
    logp.copy_(torch.where(ok, lp.gather(1, targets.long().clamp(0, V - 1)[:, None])[:, 0], 0.0))
    stats[:, 0] = z.amax(-1)
    stats[:, 1] = z.logsumexp(-1) - stats[:, 0]
    if entropy is not None:
        entropy.copy_(torch.special.entr(lp.exp()).sum(-1))
    if top_ids is not None:
        v, i = z.sort(dim=-1, descending=True, stable=True)
        n = top_ids.shape[1]
        top_ids.copy_(i[:, :n])
        top_logp.copy_(lp.gather(1, i[:, :n]))


def _logp_backward(logits, targets, stats, d_logp, d_logits, entropy=None, d_entropy=None, stream=None):
    assert d_logp.is_contiguous() and (d_entropy is None or d_entropy.is_contiguous())
    V = logits.shape[1]
    lp = logits.float() - stats[:, :1] - stats[:, 1:]
    ok = ((targets >= 0) & (targets < V)).float()
    g = (d_logp * ok)[:, None]
    d = -lp.exp() * g
    if d_entropy is not None:
        d -= d_entropy[:, None] * lp.exp() * (lp + entropy[:, None])
    d_logits.copy_(d.scatter_add_(1, targets.long().clamp(0, V - 1)[:, None], g))


@pytest.fixture(autouse=True)
def _plain(monkeypatch):
    for name, fn in (("bkmoo_embedding_forward", _embedding_forward), ("bkmoo_embedding_backward", _embedding_backward),
                     ("bkmoo_qk_norm_forward", _qk_forward), ("bkmoo_qk_norm_backward", _qk_backward),
                     ("bkmoo_token_logp_forward", _logp_forward), ("bkmoo_token_logp_backward", _logp_backward)):
        monkeypatch.setattr(native, name, fn)
    calls.clear()


def _gen(seed=0):
    return torch.Generator().manual_seed(seed)


def _close(a, b, bound):
    assert float((a.detach().double() - b.double()).norm()) <= bound * float(b.double().norm()) + 1e-30


def _places(weight, k=K):
    weight.language_grads = [torch.zeros(weight.shape, dtype=weight.dtype) for _ in range(k)]
    return weight.language_grads


def _embedding(**k):
    torch.manual_seed(1)
    return Embedding(7, 16, device="cpu", **k), torch.randint(0, 7, (2, 5), generator=_gen(2))


def _qk(dtype=torch.bfloat16):
    torch.manual_seed(2)
    layer = QueryKeyNorm(32, rotated=16, device="cpu")
    with torch.no_grad():
        for w in (layer.w_q, layer.w_k):
            w.copy_(1 + 0.2 * torch.randn(32))
    fused = torch.randn(2, 5, 6 * 32, generator=_gen(3)).to(dtype).requires_grad_()
    q, k = fused[..., :4 * 32].unflatten(-1, (4, 32)), fused[..., 4 * 32:5 * 32].unflatten(-1, (1, 32))
    return layer, fused, q, k, torch.arange(5).expand(2, 5)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_embedding_gives_the_gradient_of_the_formula(dtype):
    layer, ids = _embedding(dtype=dtype, scale=4.0)
    ids[0, 1], ids[1, 4] = -1, 7
    y = layer(ids)
    assert y.shape == (2, 5, 16) and y.dtype is dtype and bool((y[0, 1] == 0).all()) and bool((y[1, 4] == 0).all())
    c = torch.randn(2, 5, 16, generator=_gen(4)).to(dtype)
    y.backward(c)
    w = layer.weight.detach().double().requires_grad_()
    ok = ((ids >= 0) & (ids < 7))[..., None]
    (ref,) = torch.autograd.grad(w[ids.clamp(0, 6)] * 4.0 * ok, w, c.double())
    _close(layer.weight.grad, ref, torch.finfo(dtype).eps)       # two roundings of half a step


def test_embedding_apart_by_language():
    layer, ids = _embedding()
    places = _places(layer.weight)
    c = torch.randn(2, 5, 16, generator=_gen(4)).bfloat16()
    layer(ids, ROWS).backward(c.expand(2, 5, 16))
    assert layer.weight.grad is None and bool((places[1] == 0).all())
    flat, d = ids.reshape(-1), c.reshape(-1, 16).double()
    for k, (i, j) in enumerate(zip(ROWS, ROWS[1:])):
        ref = torch.zeros(7, 16, dtype=torch.float64).index_add_(0, flat[i:j], d[i:j])
        _close(places[k], ref, 2.0 ** -8)
    # a gradient whose rows are one and the same in memory
    before = [p.clone() for p in places]
    layer(ids, ROWS).backward(torch.ones(16).bfloat16().expand(2, 5, 16))
    for k, (i, j) in enumerate(zip(ROWS, ROWS[1:])):
        ref = torch.zeros(7, 16, dtype=torch.float64).index_add_(0, flat[i:j], torch.ones(j - i, 16, dtype=torch.float64))
        _close(places[k], before[k].double() + ref, 2.0 ** -8)


def test_embedding_tied_to_the_head(monkeypatch):
    """One weight that two layers use gets the sum of both gradients in every language."""
    def wgrad(dy, x, rows, dw, accumulate=False, stream=None):
        for w, i, j in zip(dw, rows, rows[1:]):
            w.copy_(w.float() + dy[i:j].float().T @ x[i:j].float())

    monkeypatch.setattr(native, "bkmoo_language_wgrad", wgrad)
    layer, ids = _embedding()
    head = LanguageLinear(16, 7, device="cpu")
    head.weight = layer.weight
    places = _places(layer.weight)
    x = torch.randn(2, 5, 16, generator=_gen(5)).bfloat16()
    (layer(ids, ROWS).float().sum() + head(x, ROWS).float().sum()).backward()
    for k, (i, j) in enumerate(zip(ROWS, ROWS[1:])):
        ref = torch.zeros(7, 16, dtype=torch.float64).index_add_(0, ids.reshape(-1)[i:j], torch.ones(j - i, 16, dtype=torch.float64))
        ref += x.reshape(-1, 16).double()[i:j].sum(0)
        assert float((places[k].double() - ref).norm()) <= 2 * 2.0 ** -8 * float(ref.norm() + 7 * (j - i))


@pytest.mark.parametrize("interleaved", [False, True])
def test_norms_give_the_gradients_of_the_formula(interleaved):
    layer, fused, q, k, pos = _qk()
    layer.interleaved = interleaved
    qo, ko = layer(q, k, pos)
    assert qo.shape == q.shape and ko.shape == k.shape
    cq, ck = torch.randn(q.shape, generator=_gen(6)).bfloat16(), torch.randn(k.shape, generator=_gen(7)).bfloat16()
    got = torch.autograd.grad((qo, ko), (fused, layer.w_q, layer.w_k), (cq, ck))
    wide = fused.detach().double().requires_grad_()
    wq, wk = (w.detach().double().requires_grad_() for w in (layer.w_q, layer.w_k))
    p = pos.reshape(-1)
    a = _normed(wide[..., :128].reshape(10, 4, 32), wq, p, layer.inv_freq, 1e-6, interleaved)
    b = _normed(wide[..., 128:160].reshape(10, 1, 32), wk, p, layer.inv_freq, 1e-6, interleaved)
    ref = torch.autograd.grad((a, b), (wide, wq, wk), (cq.reshape(a.shape).double(), ck.reshape(b.shape).double()))
    for g, r in zip(got, ref):
        _close(g, r, 2.0 ** -8)


@pytest.mark.parametrize("apart", [True, False])
@pytest.mark.parametrize("frozen", ["", "w_q", "w_k", "both"])
def test_norms_apart_by_language_and_frozen(frozen, apart):
    """What is trained gets what it gets with both trained."""
    got = []
    for freeze in ("", frozen):
        layer, fused, q, k, pos = _qk()
        for name in ("w_q", "w_k"):
            if freeze in (name, "both"):
                getattr(layer, name).requires_grad_(False)
        trained = [p for p in layer.parameters() if p.requires_grad]
        for p in trained if apart else ():
            _places(p)
        calls.clear()
        qo, ko = layer(q, k, pos, ROWS)
        (qo.float().square().sum() + ko.float().sum()).backward()
        got.append([fused.grad] + sum(((p.language_grads if apart else [p.grad]) for p in layer.parameters()
                                       if p.requires_grad and (frozen in ("", "both") or p is not getattr(layer, frozen))), []))
        assert calls == [(freeze != "both",) * 2]
        assert all(p.grad is None for p in layer.parameters() if apart or not p.requires_grad)
    n = 1 if frozen == "both" else len(got[1])
    assert all(torch.equal(u, v) for u, v in zip(got[0][:n], got[1][:n]))


def test_one_of_the_norms_is_not_apart():
    layer, fused, q, k, pos = _qk()
    both, _, q2, k2, _ = _qk()
    _places(layer.w_k)
    for m, a, b in ((layer, q, k), (both, q2, k2)):
        qo, ko = m(a, b, pos, ROWS)
        (qo.float().square().sum() + ko.float().square().sum()).backward()
    assert torch.equal(layer.w_q.grad, both.w_q.grad) and layer.w_k.grad is None
    _close(sum(g.float() for g in layer.w_k.language_grads), both.w_k.grad, 4 * 2.0 ** -8)


def test_norms_take_odd_strides_and_an_unused_result():
    layer, fused, q, k, pos = _qk()
    apart = torch.randn(10, 5, 4, 32, generator=_gen(8)).bfloat16()[::5].transpose(0, 1).contiguous().transpose(0, 1)
    assert torch.equal(layer(apart, k, pos)[0], layer(apart.contiguous(), k, pos)[0])
    qo, _ = layer(q, k, pos)
    qo.float().sum().backward()
    assert bool((layer.w_k.grad == 0).all()) and bool(torch.isfinite(fused.grad).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_log_probs_give_the_gradients_of_the_formula(dtype):
    z = torch.randn(2, 5, 13, generator=_gen(9)).to(dtype).requires_grad_()
    t = torch.randint(0, 13, (2, 5), generator=_gen(10))
    t[0, 0], t[1, 1] = -100, 13
    out = token_log_probs(z, t, entropy=True, top=3)
    assert out.logp.shape == out.entropy.shape == (2, 5) and out.top_ids.shape == out.top_logp.shape == (2, 5, 3)
    assert not out.top_logp.requires_grad and out.logp[0, 0] == 0 and out.logp[1, 1] == 0
    (out.logp.sum() * -0.5 + 0.1 * out.entropy.sum()).backward()
    w = z.detach().double().requires_grad_()
    lp = w.log_softmax(-1)
    # the stand-in's own fp32: |log p| is at most 8 here, off by three roundings of it, and that is p's
    # relative error; six more of products and sums
    assert float(lp.detach().abs().max()) <= 8
    bound = torch.finfo(dtype).eps + (3 * 8 + 6) * 2.0 ** -24
    ok = (t >= 0) & (t < 13)
    loss = -0.5 * (lp.gather(-1, t.clamp(0, 12)[..., None])[..., 0] * ok).sum() - 0.1 * (lp.exp() * lp).sum()
    (ref,) = torch.autograd.grad(loss, w, retain_graph=True)
    _close(z.grad, ref, bound)
    # entropy alone; logp alone; neither
    for entropy, pick in ((True, 1), (False, 0)):
        z.grad = None
        token_log_probs(z, t, entropy=entropy)[pick].sum().backward()
        what = -(lp.exp() * lp).sum() if pick else (lp.gather(-1, t.clamp(0, 12)[..., None])[..., 0] * ok).sum()
        (ref,) = torch.autograd.grad(what, w, retain_graph=True)
        _close(z.grad, ref, bound)
    plain = token_log_probs(z.detach(), t)
    assert plain.entropy is None and plain.top_ids is None and plain.top_logp is None and not plain.logp.requires_grad


def test_refusals():
    layer, fused, q, k, pos = _qk()
    with pytest.raises(ValueError, match="same tokens"):
        layer(q, k, torch.arange(5))
    with pytest.raises(ValueError, match="same tokens"):
        layer(q, k[:1], pos)
    with pytest.raises(ValueError, match="one target"):
        token_log_probs(torch.zeros(2, 5, 13), torch.zeros(10, dtype=torch.int64))
    emb, ids = _embedding()
    _places(emb.weight)
    with pytest.raises(ValueError, match="bounds of the 3 languages"):
        emb(ids, [0, 4, 10]).float().sum().backward()


@pytest.mark.parametrize("make", ["embedding", "norm", "logp"])
def test_gradients_of_gradients_are_refused(make):
    if make == "embedding":
        layer, ids = _embedding()
        y, x = layer(ids), layer.weight
    elif make == "norm":
        layer, x, q, k, pos = _qk()
        y = layer(q, k, pos)[0]
    else:
        x = torch.randn(2, 13, requires_grad=True)
        y = token_log_probs(x, torch.tensor([1, 2])).logp
    (g,) = torch.autograd.grad(y.float().square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        g.float().square().sum().backward()


def test_the_norms_layer_can_be_saved():
    layer, _, q, k, pos = _qk()
    other = pickle.loads(pickle.dumps(layer))
    assert torch.equal(other(q, k, pos)[0], layer(q, k, pos)[0])
    assert list(other.inv_freq) == [10000.0 ** (-i / 8) for i in range(8)] and math.isclose(other.inv_freq[0], 1.0)


class _Stream:
    notes = []

    def __init__(self, name):
        self.cuda_stream = name

    def wait_stream(self, other):
        self.notes.append((self.cuda_stream, "waits for", other.cuda_stream))


@pytest.mark.parametrize("which", ["embedding", "norm"])
def test_gradients_written_on_another_stream(monkeypatch, which):
    """As for the other layers: the write is ordered against the stream of begin_batch()."""
    from paper_2606_05613_gb300.hook import LanguageGrads
    home, now = _Stream("home"), _Stream("other")
    monkeypatch.setattr(_Stream, "notes", [])
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: now)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: now.cuda_stream, raising=False)
    name = "bkmoo_embedding_backward" if which == "embedding" else "bkmoo_qk_norm_backward"
    real = getattr(native, name)

    def noted(*a, **k):
        _Stream.notes.append("write")
        return real(*a, **k)

    monkeypatch.setattr(native, name, noted)
    if which == "embedding":
        layer, ids = _embedding()
        y = layer(ids, ROWS)
    else:
        layer, _, q, k, pos = _qk()
        y = layer(q, k, pos, ROWS)[0]
    for p in layer.parameters():
        p.language_grads = LanguageGrads([torch.zeros(p.shape, dtype=torch.bfloat16) for _ in range(K)], home, 0)
    y.float().sum().backward()
    notes = [n for i, n in enumerate(_Stream.notes) if i == 0 or n != _Stream.notes[i - 1]]
    assert notes == [("other", "waits for", "home"), "write", ("home", "waits for", "other")]
