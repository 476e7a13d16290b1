"""Calls of the embedding, the norms and the log probabilities on two streams at once, eager and
replayed: each has its own workspace, and the results are those of one call after the other."""
import pytest
import torch

from paper_2606_05613_gb300 import native as bk

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16


class _Work:
    def __init__(self, seed, T=3000, V=2000, D=264, hd=64, vocab=20011):
        g = torch.Generator(device=DEV).manual_seed(seed)

        def normal(*shape):
            return torch.randn(*shape, generator=g, device=DEV).to(BF)

        self.ids = torch.randint(-1, V, (T,), generator=g, device=DEV)
        self.rows = [0, T // 3, T // 3, T]
        self.table, self.dy = normal(V, D), normal(T, D)
        self.q, self.k, self.dqo, self.dko = normal(T, 6, hd), normal(T, 2, hd), normal(T, 6, hd), normal(T, 2, hd)
        self.w, self.pos, self.freq = [normal(hd), normal(hd)], torch.arange(T, device=DEV), bk.rope_frequencies(hd, 1e4)
        self.z, self.t = normal(300, vocab), torch.randint(0, vocab, (300,), generator=g, device=DEV)
        self.one, self.t1 = normal(1, 8 * vocab), torch.randint(0, vocab, (1,), generator=g, device=DEV)
        self.g = torch.randn(300, generator=g, device=DEV)
        self.out = [torch.empty(T, D, dtype=BF, device=DEV)] + [torch.empty(V, D, device=DEV) for _ in range(3)]
        self.norm = [torch.empty_like(x) for x in (self.q, self.k, self.q, self.k)]
        self.dw = [torch.empty(hd, device=DEV) for _ in range(6)]
        self.top = [torch.empty(300, device=DEV), torch.empty(300, 2, device=DEV), torch.empty(300, device=DEV),
                    torch.empty(300, 9, dtype=torch.int64, device=DEV), torch.empty(300, 9, device=DEV), torch.empty_like(self.z)]
        self.first = [torch.empty(1, device=DEV), torch.empty(1, 20, dtype=torch.int64, device=DEV), torch.empty(1, 20, device=DEV)]

    def run(self):
        bk.bkmoo_embedding_forward(self.table, self.ids, self.out[0], scale=2.0)
        bk.bkmoo_embedding_backward(self.dy, self.ids, self.rows, self.out[1:], scale=2.0)
        bk.bkmoo_qk_norm_forward(self.q, self.k, *self.w, self.pos, self.freq, *self.norm[:2])
        bk.bkmoo_qk_norm_backward(self.dqo, self.dko, self.q, self.k, *self.w, self.pos, self.freq, self.rows, *self.norm[2:],
                                  self.dw[:3], self.dw[3:])
        bk.bkmoo_token_logp_forward(self.z, self.t, *self.top[:5])
        bk.bkmoo_token_logp_backward(self.z, self.t, self.top[1], self.g, self.top[5], self.top[2], self.g)
        bk.bkmoo_token_logp_forward(self.one, self.t1, self.first[0], None, None, *self.first[1:])

    def results(self):
        return [t.clone() for t in self.out + self.norm + self.dw + self.top + self.first]

    def clear(self):
        for t in self.out + self.norm + self.dw + self.top + self.first:
            t.zero_()


@pytest.mark.parametrize("replayed", [False, True])
def test_two_streams_at_once(replayed):
    work = [_Work(1), _Work(2)]
    want = []
    for w in work:
        w.run()
        want.append(w.results())
    streams = [torch.cuda.Stream() for _ in work]
    runs = [w.run for w in work]
    if replayed:
        graphs = [torch.cuda.CUDAGraph() for _ in work]
        for g, w in zip(graphs, work):
            with torch.cuda.graph(g):
                w.run()
        runs = [g.replay for g in graphs]
    for w in work:
        w.clear()
    torch.cuda.synchronize()
    for _ in range(20):
        for s, run in zip(streams, runs):
            with torch.cuda.stream(s):
                run()
    torch.cuda.synchronize()
    for w, r in zip(work, want):
        assert all(torch.equal(a, b) for a, b in zip(w.results(), r))
