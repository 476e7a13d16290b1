"""The layers of a language model together on the GPU: embedding, projections, norms of queries
and keys, log probabilities; gradients apart by language, another stream, a captured step, and
the example that trains such a model."""
import importlib.util
import os

import pytest
import torch

from paper_2606_05613_gb300 import native as bk
from paper_2606_05613_gb300.hook import BucketMOO
from paper_2606_05613_gb300.language import Embedding, LanguageLinear, QueryKeyNorm, token_log_probs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROWS = [0, 37, 37, 150]
K, V, D, H, HD = 3, 1003, 72, 3, 48
# bf16 results behind one another: 2^-9 each in the 2-norm (a rounding is at most 2^-9 of its value's
# binade, uniformly), at most ten of them on the way to a gradient (x, projection, norm, sum, logits; their
# gradients; the weight's)
TOL = 10 * 2.0 ** -9


class _Model(torch.nn.Module):
    def __init__(self, seed=0):
        super().__init__()
        torch.manual_seed(seed)
        self.embedding = Embedding(V, D, scale=2.0)
        self.project = LanguageLinear(D, 2 * H * HD)
        self.norm = QueryKeyNorm(HD, rotated=32)
        self.head = LanguageLinear(H * HD, V)
        with torch.no_grad():
            for w in (self.norm.w_q, self.norm.w_k):
                w.add_(0.2 * torch.randn(HD, device=DEV))

    def forward(self, ids, pos, rows):
        q, k = self.project(self.embedding(ids, rows), rows).unflatten(-1, (2 * H, HD)).split(H, -2)
        q, k = self.norm(q, k, pos, rows)
        return self.head((q + k).flatten(-2), rows)


def _plain(m, ids, pos):
    """The same by elementary operations, in 64 bits."""
    e, p, wq, wk, h = (w.double() for w in (m.embedding.weight, m.project.weight, m.norm.w_q, m.norm.w_k, m.head.weight))
    x = e[ids.clamp(0, V - 1)] * 2.0 * ((ids >= 0) & (ids < V))[:, None]
    a = pos.double()[:, None] * torch.tensor([10000.0 ** (-i / 16) for i in range(16)], dtype=torch.float64, device=DEV)
    y = (x @ p.T).unflatten(-1, (2, H, HD))
    y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + 1e-6) * torch.stack([wq, wk])[:, None]
    u, v, c, s = y[..., :16], y[..., 16:32], a.cos()[:, None, None], a.sin()[:, None, None]
    y = torch.cat([u * c - v * s, v * c + u * s, y[..., 32:]], -1)
    return y.sum(1).flatten(-2) @ h.T


def _loss(logits, targets, c):
    out = token_log_probs(logits, targets, entropy=True)
    return (c * (out.logp + 0.1 * out.entropy)).sum()


def _plain_loss(logits, targets, c):
    lp = logits.log_softmax(-1)
    t = torch.where((targets >= 0) & (targets < V), lp.gather(1, targets.clamp(0, V - 1)[:, None])[:, 0], 0.0)
    return (c.double() * (t - 0.1 * (lp.exp() * lp).sum(-1))).sum()


def _batch(seed=1):
    g = torch.Generator(device=DEV).manual_seed(seed)
    ids = torch.randint(0, V, (ROWS[-1],), generator=g, device=DEV)
    targets = torch.randint(0, V, (ROWS[-1],), generator=g, device=DEV)
    ids[5], targets[:9], targets[100] = -1, -100, V
    return ids, torch.randint(0, 100000, (ROWS[-1],), generator=g, device=DEV), targets, torch.randn(ROWS[-1], generator=g, device=DEV)


def _relative(a, b):
    a, b = a.detach().double(), b.detach().double()
    return float((a - b).norm() / b.norm())


def test_gradients_come_apart_by_language():
    m = _Model()
    params = list(m.parameters())
    moo = BucketMOO(params, K, 1 << 14, rule="mean")
    ids, pos, targets, c = _batch()
    moo.begin_batch()
    logits = m(ids, pos, ROWS)
    assert _relative(logits, _plain(m, ids, pos)) <= TOL
    _loss(logits, targets, c).backward()
    for k, (i, j) in enumerate(zip(ROWS, ROWS[1:])):
        if i == j:
            assert all(bool((p.language_grads[k] == 0).all()) for p in params)
            continue
        ref = torch.autograd.grad(_plain_loss(_plain(m, ids[i:j], pos[i:j]), targets[i:j], c[i:j]), params)
        for p, r in zip(params, ref):
            assert _relative(p.language_grads[k], r) <= TOL
    grads = [g.clone() for g in moo.grads]
    d = moo.finish()
    out = torch.empty_like(d)
    bk.Resolver(K, torch.bfloat16, moo.layout.offsets, DEV).resolve(grads, "mean", out)
    assert torch.equal(d, out)


def test_without_languages_the_ordinary_gradient():
    m = _Model()
    params = list(m.parameters())
    ids, pos, targets, c = _batch()
    _loss(m(ids, pos, None), targets, c).backward()
    ref = torch.autograd.grad(_plain_loss(_plain(m, ids, pos), targets, c), params)
    for p, r in zip(params, ref):
        assert _relative(p.grad, r) <= TOL


def test_two_passes_add_up():
    m = _Model()
    moo = BucketMOO(m.parameters(), K, 1 << 14)
    ids, pos, targets, c = _batch()
    moo.begin_batch()
    _loss(m(ids, pos, ROWS), targets, c).backward()
    once = [g.clone() for g in moo.grads]
    moo.begin_batch()
    for _ in range(2):
        _loss(m(ids, pos, ROWS), targets, c).backward()
    for a, b in zip(once, moo.grads):
        assert torch.equal(a * 2, b)              # a power of two: exact in bf16
    moo.finish()


@pytest.mark.parametrize("frozen", ["norm.w_q", "norm.w_k", "embedding.weight"])
def test_weights_that_are_frozen(frozen):
    m, free = _Model(), _Model()
    dict(m.named_parameters())[frozen].requires_grad_(False)
    got = []
    ids, pos, targets, c = _batch()
    for model in (m, free):
        moo = BucketMOO(model.parameters(), K, 1 << 14)
        moo.begin_batch()
        _loss(model(ids, pos, ROWS), targets, c).backward()
        got.append({n: [g.clone() for g in p.language_grads] for n, p in model.named_parameters() if p.requires_grad})
        moo.finish()
    assert set(got[0]) == set(got[1]) - {frozen}
    assert all(torch.equal(u, v) for n in got[0] for u, v in zip(got[0][n], got[1][n]))


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
    m = _Model()
    moo = BucketMOO(m.parameters(), K, 1 << 14, rule="mean")
    ids, pos, targets, c = _batch()
    other = torch.cuda.Stream()

    def run(stream):
        moo.begin_batch()
        if stream is None:
            _loss(m(ids, pos, ROWS), targets, c).backward()
        else:
            stream.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(stream):
                loss = _loss(_Late.apply(m(ids, pos, ROWS)), targets, c)
            loss.backward()
        return moo.finish().clone(), [g.clone() for g in moo.grads]

    d, grads = run(None)
    for _ in range(2):
        late, late_grads = run(other)
        assert torch.equal(d, late) and all(torch.equal(u, v) for u, v in zip(grads, late_grads))
    torch.cuda.synchronize()


def test_a_captured_pass():
    """Forward and backward pass in a graph: a replay on another batch gives that batch's gradients
    of an eager pass, bit for bit."""
    m = _Model()
    places = {}
    for n, p in m.named_parameters():
        places[n] = p.language_grads = [torch.zeros(p.shape, dtype=p.dtype, device=DEV) for _ in range(K)]
    batch = _batch()

    def step():
        for ps in places.values():
            for g in ps:
                g.zero_()
        _loss(m(batch[0], batch[1], ROWS), batch[2], batch[3]).backward()

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (1, 2):
        for t, new in zip(batch, _batch(seed)):
            t.copy_(new)
        graph.replay()
        got = {n: [g.clone() for g in ps] for n, ps in places.items()}
        step()
        assert all(torch.equal(u, v) for n in got for u, v in zip(got[n], places[n]))


def test_steps_with_a_captured_pass():
    """begin_batch(), a replay on its stream and finish(): the directions of eager steps, bit for bit."""
    m = _Model()
    moo = BucketMOO(m.parameters(), K, 1 << 14, rule="mean")
    batch, stream = _batch(), torch.cuda.Stream()
    want = []
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for seed in (1, 2, 3):
            moo.begin_batch()
            new = _batch(seed)
            _loss(m(new[0], new[1], ROWS), new[2], new[3]).backward()
            want.append(moo.finish().clone())
        moo.begin_batch()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            _loss(m(batch[0], batch[1], ROWS), batch[2], batch[3]).backward()
        for seed, d in zip((1, 2, 3), want):
            for t, new in zip(batch, _batch(seed)):
                t.copy_(new)
            moo.begin_batch()
            graph.replay()
            assert torch.equal(moo.finish(), d)
    torch.cuda.synchronize()


def _example():
    spec = importlib.util.spec_from_file_location("multilingual_lm_step", os.path.join(ROOT, "examples", "multilingual_lm_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("rule", ["mgda", "cagrad"])
def test_the_example_runs(rule):
    losses = _example().run(steps=3, K=3, rule=rule)
    assert losses.shape == (3, 3) and bool(torch.isfinite(losses).all())


def test_the_examples_gradients():
    """Each language's gradient in a batch of all is that of a pass over its sequences alone.  At
    most 40 bf16 results lie behind one another in two layers, forwards and backwards, off by 2^-9 each
    in the 2-norm on either side."""
    ex = _example()
    torch.manual_seed(0)
    m = ex.Model(97, 64, 160, 2, 4, 2, 16)
    each, S = [3, 0, 5], 20
    data = ex.sequences(3, each, S, 97)
    ids, targets = data[:, :-1].contiguous(), data[:, 1:].contiguous()
    pos = torch.arange(S, device=DEV).expand(ids.shape)
    rows = [0, 3 * S, 3 * S, 8 * S]
    moo = BucketMOO(m.parameters(), 3, 1 << 16)
    moo.begin_batch()
    token_log_probs(m(ids, pos, rows), targets).logp.sum().backward()
    together = {n: [g.clone() for g in p.language_grads] for n, p in m.named_parameters()}
    moo.finish()
    first = 0
    for k, n in enumerate(each):
        if n == 0:
            assert all(bool((g[k] == 0).all()) for g in together.values())
            continue
        for p in m.parameters():
            p.grad = None
        token_log_probs(m(ids[first:first + n], pos[first:first + n], None), targets[first:first + n]).logp.sum().backward()
        for name, p in m.named_parameters():
            assert _relative(together[name][k], p.grad) <= 2 * 40 * 2.0 ** -9, name
        first += n
