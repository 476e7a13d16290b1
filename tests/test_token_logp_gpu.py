"""Log probabilities of tokens, entropies, most likely tokens and the gradient of the logits
against the formula in 64 bits, on the GPU."""
import math

import pytest
import torch

from paper_2606_05613_gb300 import native as bk

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24                                   # a rounding to fp32, relative
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
BF, F32 = torch.bfloat16, torch.float32
INF = math.inf


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _logits(T, V, dtype, seed, ld=None, ahead=0, std=2.0):
    ld = V if ld is None else ld
    room = torch.full((ahead + T * ld,), 7.0, dtype=dtype, device=DEV)
    z = room[ahead:].view(T, ld)[:, :V]
    z.copy_(torch.randn(T, V, generator=_gen(seed), device=DEV) * std)
    return z, room


def _targets(T, V, seed, dtype=torch.int64):
    t = torch.randint(0, V, (T,), generator=_gen(seed), device=DEV)
    if T > 3:
        t[1], t[T // 2] = -100, V
    return t.to(dtype)


def _forward(z, targets, top=0):
    T = z.shape[0]
    out = [torch.full((T,), 9.0, device=DEV), torch.full((T, 2), 9.0, device=DEV), torch.full((T,), 9.0, device=DEV), None,
           None]
    if top:
        out[3] = torch.full((T, top), -9, dtype=torch.int64, device=DEV)
        out[4] = torch.full((T, top), 9.0, device=DEV)
    bk.bkmoo_token_logp_forward(z, targets, *out)
    return out


class _Ref:
    """The formula in 64 bits for rows with a finite logit, and bounds on fp32's errors."""

    def __init__(self, z, targets):
        T, V = z.shape
        d = z.double()
        self.ok = (targets >= 0) & (targets < V)
        self.at = targets.long().clamp(0, V - 1)[:, None]
        self.m = d.max(-1).values
        x = d - self.m[:, None]
        e = torch.exp(x)
        s = e.sum(-1)
        self.L = torch.log(s)
        self.lp = x - self.L[:, None]
        self.p = torch.exp(self.lp)
        low = torch.where(self.p > 0, x, 0.0)
        far = -(self.p * low).sum(-1)                     # mean distance from the maximum
        self.H = self.L + far
        self.logp = torch.where(self.ok, torch.gather(self.lp, 1, self.at)[:, 0], 0.0)
        # s: an element's exponent is off by 3 roundings of |x|, 2^. by 2 units in the last place; a
        # thread's part of the row by an addition each and as many changes of base; 60 to join them
        self.s_err = U * (3 * far + 4 + 3 * (V / 256 + 8) + 60)
        self.L_err = self.s_err + U * 2 * self.L.abs()
        self.lp_err = self.L_err[:, None] + U * 2 * (x.abs() + self.lp.abs())
        # u: the same of the sum of e x, in which a change of base by d moves s d
        square = (self.p * low.square()).sum(-1)
        self.H_err = self.L_err + self.s_err * (far + 1) * 3 + U * 6 * (square + far + self.L.abs())

    def check(self, out, z):
        logp, stats, H, ids, top = out
        err = torch.gather(self.lp_err, 1, self.at)[:, 0]
        assert bool(((logp.double() - self.logp).abs() <= 1.01 * torch.where(self.ok, err, 0.0)).all())
        assert torch.equal(stats[:, 0].double(), self.m)
        assert bool(((stats[:, 1].double() - self.L).abs() <= 1.01 * self.L_err).all())
        assert bool(((H.double() - self.H).abs() <= 1.01 * self.H_err).all())
        if ids is not None:
            n = ids.shape[1]
            want = torch.sort(z.float(), stable=True, dim=-1, descending=True).indices[:, :n]
            assert torch.equal(ids, want)
            got, ref, err = top.double(), torch.gather(self.lp, 1, ids), torch.gather(self.lp_err, 1, ids)
            # 3e38 below the maximum by 6e38: log p, -6e38, is beyond fp32's largest, 3.4e38, so it rounds
            # to minus infinity
            ref = torch.where(ref < -torch.finfo(F32).max, -INF, ref)
            dead = ref == -INF
            assert bool(((got == ref) | ~dead).all())
            assert bool((dead | ((got - ref).abs() <= 1.01 * err)).all())

    def check_grad(self, dz, g, h):
        g = torch.where(self.ok, g.double(), 0.0)[:, None]
        h = torch.zeros_like(g) if h is None else h.double()[:, None]
        lp = self.lp.clamp(min=-1e5)
        ref = -self.p * (g + h * (lp + self.H[:, None]))
        ref.scatter_add_(1, self.at, g)
        # p by the error of log p, of its exponent's product and 2^.
        p_err = torch.where(self.p > 0, self.lp_err + U * (3 * lp.abs() + 4), 0.0)
        err = self.p * (p_err * (g.abs() + h.abs() * (lp.abs() + self.H[:, None])) +
                        h.abs() * (self.lp_err.clamp(max=1e5) + self.H_err[:, None]) +
                        4 * U * (g.abs() + h.abs() * (lp.abs() + self.H[:, None])))
        err.scatter_add_(1, self.at, U * g.abs())
        err += 2.0 ** -126                                # results and probabilities below the normal numbers
        assert bool(((dz.double() - ref).abs() <= 1.01 * (err + HALF[dz.dtype] * (ref.abs() + err))).all())


SHAPES = [
    # T, V, ld beyond V, elements ahead, n
    (1, 1, 0, 0, 1), (1, 2, 0, 0, 2), (3, 7, 0, 0, 7), (5, 31, 1, 1, 20), (4, 33, 0, 3, 32), (2, 500, 0, 0, 32),
    (7, 1001, 0, 0, 5), (9, 1000, 24, 0, 5), (3, 4096, 0, 0, 20), (1, 8191, 0, 1, 1), (1, 8192, 0, 0, 20), (2, 16391, 3, 5, 32),
    (1, 65536, 0, 0, 20), (1, 151936, 0, 0, 20), (5, 50257, 0, 0, 5), (31, 32000, 0, 0, 20), (700, 10007, 0, 0, 3),
    (160, 33000, 0, 7, 8), (1300, 8200, 8, 0, 0), (2, 262147, 0, 0, 32),
]


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("T,V,beyond,ahead,n", SHAPES)
def test_forward(T, V, beyond, ahead, n, dtype):
    z, _ = _logits(T, V, dtype, 1, V + beyond, ahead)
    targets = _targets(T, V, 2, torch.int32 if V % 2 else torch.int64)
    ref = _Ref(z, targets)
    out = _forward(z, targets, n)
    ref.check(out, z)
    # what is not asked for is not needed
    logp = torch.empty(T, device=DEV)
    bk.bkmoo_token_logp_forward(z, targets, logp)
    assert bool(((logp - out[0]).double().abs() <= 2.02 * torch.gather(ref.lp_err, 1, ref.at)[:, 0]).all())
    again = _forward(z, targets, n)
    assert all(torch.equal(a, b) for a, b in zip(out, again) if a is not None)


@pytest.mark.parametrize("entropy", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("T,V,beyond,ahead,n", SHAPES)
def test_backward(T, V, beyond, ahead, n, dtype, entropy):
    z, _ = _logits(T, V, dtype, 3, V + beyond, ahead)
    targets = _targets(T, V, 4)
    ref = _Ref(z, targets)
    _, stats, H, *_ = _forward(z, targets)
    g = torch.randn(T, generator=_gen(5), device=DEV)
    h = torch.randn(T, generator=_gen(6), device=DEV) * 0.1 if entropy else None
    if T > 8:
        g[5] = 0.0
        if entropy:
            h[5] = 0.0
    # rows that start at another place of 16 bytes than the logits', and at the same
    for more in (0, 1):
        dz, room = _logits(T, V, dtype, 7, V + beyond + more, ahead + more)
        bk.bkmoo_token_logp_backward(z, targets, stats, g, dz, H if entropy else None, h)
        ref.check_grad(dz, g, h)
        assert int((room == 7.0).sum()) >= room.numel() - T * V
    # in the logits' place: the same bits
    same = torch.as_strided(torch.cat([z.new_zeros(ahead), torch.zeros(T * (V + beyond), dtype=dtype, device=DEV)]),
                            (T, V), (V + beyond, 1), ahead).copy_(z)
    bk.bkmoo_token_logp_backward(same, targets, stats, g, same, H if entropy else None, h)
    assert torch.equal(same, dz)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("T,V", [(3, 40), (2, 5000), (1, 70000), (800, 700)])
def test_equal_logits(T, V, dtype):
    """Ties go to the lowest index, also where more are equal than a list holds."""
    z = torch.full((T, V), 1.5, dtype=dtype, device=DEV)
    z[:, V // 2] = 2.0
    z[:, V // 3] = 0.0
    z[:, V // 4] = -0.0
    targets = _targets(T, V, 2)
    _Ref(z, targets).check(_forward(z, targets, 32), z)
    z = (torch.arange(V, device=DEV) % 3).to(dtype).expand(T, V).contiguous()
    _Ref(z, targets).check(_forward(z, targets, 32), z)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("V", [300, 70001])
def test_the_likely_ones_lie_close_together(V, dtype):
    """Rising, falling and clustered logits: the best ones with one thread or with all."""
    rise = torch.arange(V, device=DEV, dtype=torch.float32)
    z = torch.stack([rise, -rise, torch.where((rise > 99) & (rise < 180), rise, -rise), rise % 256, -(rise % 2048)])
    z = (z * (20.0 / V)).to(dtype)
    targets = torch.arange(5, device=DEV) * 50
    _Ref(z, targets).check(_forward(z, targets, 32), z)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("V", [12, 1001, 70000])
def test_masked_logits(V, dtype):
    """Tokens that are ruled out by minus infinity or by the type's lowest value; rows of which
    little or nothing is left."""
    z, _ = _logits(8, V, dtype, 1)
    lowest = torch.finfo(dtype).min
    z[0, ::2] = -INF
    z[1, 1:] = -INF
    z[2, :-1] = -INF
    z[3] = lowest
    z[4, ::3] = lowest
    z[5, : V // 2] = -INF
    z[5, V // 2:] = lowest
    z[6] = 3e38                                     # nothing overflows
    z[6, 0] = -3e38
    targets = torch.tensor([1, 0, V - 1, 5, 1, V - 1, 3, -1], device=DEV)
    ref = _Ref(z, targets)
    out = _forward(z, targets, min(V, 32))
    ref.check(out, z)
    g, h = torch.randn(8, generator=_gen(2), device=DEV), torch.randn(8, generator=_gen(3), device=DEV)
    for hh in (None, h):
        dz = torch.empty_like(z)
        bk.bkmoo_token_logp_backward(z, targets, out[1], g, dz, None if hh is None else out[2], hh)
        ref.check_grad(dz, g, hh)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("T,V", [(2, 300), (3, 5000), (2, 151936), (700, 12007)])
def test_few_tokens_are_allowed(T, V, dtype):
    """A grammar leaves 0 to 60 tokens of a row, the others are minus infinity or the lowest value."""
    z, _ = _logits(T, V, dtype, 1)
    left = torch.rand(T, V, generator=_gen(2), device=DEV).argsort(-1) < torch.tensor([3, 19, 33, 60, 1], device=DEV)[
        torch.arange(T, device=DEV) % 5][:, None]
    targets = left.float().argmax(-1)
    for mask in (-INF, torch.finfo(dtype).min):
        y = torch.where(left, z, mask).to(dtype)
        _Ref(y, targets).check(_forward(y, targets, 20), y)
        y[:, V // 2:] = z[:, V // 2:V // 2 + 1]             # and half of them all alike
        _Ref(y, targets).check(_forward(y, targets, 32), y)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("V", [12, 1001, 70000])
def test_rows_without_a_token_and_rows_that_are_no_numbers(V, dtype):
    z, _ = _logits(6, V, dtype, 1)
    z[0] = -INF
    z[1] = -INF
    z[2, V // 2] = math.nan
    z[3, V // 2] = INF
    z[4] = -INF
    z[4, 3] = math.nan
    targets = torch.tensor([3, -1, 1, 1, 1, 2], device=DEV)
    n = min(V, 32)
    logp, stats, H, ids, top = _forward(z, targets, n)
    assert logp[0] == -INF and logp[1] == 0 and bool((H[:2] == 0).all())
    assert bool((top[:2] == -INF).all()) and torch.equal(ids[0], torch.arange(n, device=DEV))
    assert bool(torch.isnan(logp[2:5]).all()) and bool(torch.isnan(H[2:5]).all()) and bool(torch.isnan(top[2:5]).all())
    assert int(ids[3, 0]) == V // 2                 # plus infinity is the largest, NaN below all
    assert int(ids[4, 0]) == 0 and (V > n or int(ids[4, -1]) == 3) and (V > n or int(ids[2, -1]) == V // 2)
    assert all(len(set(r)) == n and min(r) >= 0 and max(r) < V for r in ids.tolist())
    fine = _Ref(z[5:], targets[5:])
    fine.check([logp[5:], stats[5:], H[5:], ids[5:], top[5:]], z[5:])
    g, h = torch.ones(6, device=DEV), torch.ones(6, device=DEV)
    for hh in (None, h):
        dz = torch.empty_like(z)
        bk.bkmoo_token_logp_backward(z, targets, stats, g, dz, None if hh is None else H, hh)
        assert bool((dz[:2] == 0).all()) and bool(torch.isnan(dz[2:5]).all())
        fine.check_grad(dz[5:], g[5:], None if hh is None else hh[5:])


def test_rows_that_count_for_nothing_are_not_read():
    T, V = 20, 999
    z = torch.full((T, V), math.nan, device=DEV)
    targets = torch.full((T,), -1, device=DEV)
    dz = torch.ones(T, V, device=DEV)
    bk.bkmoo_token_logp_backward(z, targets, torch.zeros(T, 2, device=DEV), torch.full((T,), math.nan, device=DEV), dz)
    assert bool((dz == 0).all())


def test_gradients_are_those_of_differences():
    V, h = 37, 1e-4
    z, _ = _logits(1, V, F32, 1)
    targets = torch.tensor([5], device=DEV)
    _, stats, H, *_ = _forward(z, targets)
    g, e = torch.tensor([1.5], device=DEV), torch.tensor([0.5], device=DEV)
    dz = torch.empty_like(z)
    bk.bkmoo_token_logp_backward(z, targets, stats, g, dz, H, e)

    def f(d):
        lp = torch.log_softmax(d, -1)
        return float(1.5 * lp[0, 5] - 0.5 * (lp.exp() * lp).sum())

    for v in (0, 5, 20, 36):
        hi, lo = z.double(), z.double()
        hi[0, v] += h
        lo[0, v] -= h
        # h^2 of the third derivative, fp64's rounding over h, and fp32's of the gradient
        assert abs(float(dz[0, v]) - (f(hi) - f(lo)) / (2 * h)) <= 2e-6


def test_rows_beyond_32_bits():
    T, V, ld = 10, 5001, 1 << 29
    room = torch.empty((T - 1) * ld + V, dtype=BF, device=DEV)
    z = torch.as_strided(room, (T, V), (ld, 1))
    z.copy_(torch.randn(T, V, generator=_gen(1), device=DEV))
    targets = _targets(T, V, 2)
    ref = _Ref(z, targets)
    out = _forward(z, targets, 20)
    ref.check(out, z)
    g = torch.randn(T, generator=_gen(3), device=DEV)
    bk.bkmoo_token_logp_backward(z, targets, out[1], g, z)
    ref.check_grad(z, g, None)


def test_no_rows():
    z = torch.empty(0, 50, device=DEV)
    targets, none = torch.empty(0, dtype=torch.int64, device=DEV), torch.empty(0, device=DEV)
    bk.bkmoo_token_logp_forward(z, targets, none)
    bk.bkmoo_token_logp_backward(z, targets, torch.empty(0, 2, device=DEV), none, z.clone())


def test_captured_and_replayed_and_on_another_stream():
    T, V = 37, 20000
    z, _ = _logits(T, V, BF, 1)
    targets = _targets(T, V, 2)
    out = _forward(z, targets, 20)
    g, h = torch.randn(T, device=DEV), torch.randn(T, device=DEV)
    dz = torch.empty_like(z)

    def step(stream=None):
        bk.bkmoo_token_logp_forward(z, targets, *out, stream=stream)
        bk.bkmoo_token_logp_backward(z, targets, out[1], g, dz, out[2], h, stream=stream)

    step()
    want = [t.clone() for t in out + [dz]]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for t in out + [dz]:
            t.zero_()
    step(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, out + [dz]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    z.copy_(torch.randn(T, V, generator=_gen(30), device=DEV))
    targets.copy_(_targets(T, V, 31))
    graph.replay()
    ref = _Ref(z, targets)
    ref.check(out, z)
    ref.check_grad(dz, g, h)
