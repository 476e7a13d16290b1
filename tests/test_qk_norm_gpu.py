"""Norms of queries and keys with the rotation, and their gradients apart by language, against
the formula in 64 bits, on the GPU."""
import math

import pytest
import torch

from paper_2606_05613_gb300 import native as bk

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24                                   # a rounding to fp32, relative
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
BF = torch.bfloat16


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _normal(*shape, seed, std=1.0):
    return torch.randn(*shape, generator=_gen(seed), device=DEV) * std


def _fused(T, hq, hk, hd, seed, ld=None, std=1.0):
    """Queries and keys as columns of one matrix with rows of `ld`, and the matrix; what is
    neither holds 7."""
    width = (hq + hk) * hd
    room = torch.full((max(T, 1), ld or width), 7.0, dtype=BF, device=DEV)
    room[:T, :width] = _normal(T, width, seed=seed, std=std)
    q = room[:T, :hq * hd].view(T, hq, hd) if T else room.new_empty(0, hq, hd)
    k = room[:T, hq * hd:width].view(T, hk, hd) if T else room.new_empty(0, hk, hd)
    return q, k, room


def _turns(pos, freq, back):
    a = pos.double()[:, None] * torch.tensor(list(freq), dtype=torch.float64, device=DEV)
    return torch.polar(torch.ones_like(a), -a if back else a)[:, None]


def _pairs(x, rot, interleaved):
    z = x[..., :rot]
    return z.unflatten(-1, (rot // 2, 2)) if interleaved else z.unflatten(-1, (2, rot // 2)).transpose(-1, -2)


def _unpairs(z, interleaved):
    return z.flatten(-2) if interleaved else z.transpose(-1, -2).flatten(-2)


def _rotate(x, turn, rot, interleaved):
    if rot == 0:
        return x
    z = torch.view_as_complex(_pairs(x, rot, interleaved).contiguous()) * turn
    return torch.cat([_unpairs(torch.view_as_real(z), interleaved), x[..., rot:]], -1)


def _size(x, rot, interleaved):
    """An element's size under any rotation: |a| + |b| of its pair."""
    z = _pairs(x.abs(), rot, interleaved).sum(-1, keepdim=True).expand(*x.shape[:-1], rot // 2, 2)
    return torch.cat([_unpairs(z, interleaved), x[..., rot:].abs()], -1)


def _reference(x, w, do, pos, freq, eps, interleaved):
    """Results and bounds on fp32's part of the errors: out, its bound; dx, its bound; every
    row's and head's part of dw, and its size."""
    hd, rot = x.shape[-1], 2 * len(freq)
    x, w, do = x.double(), w.double(), do.double()
    r = 1 / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
    n = x * r
    out = _rotate(n * w, _turns(pos, freq, False), rot, interleaved)
    # r: hd additions of squares, under a root (half of them), its own error of 2 units, 1 / hd, eps;
    # an angle is off by 2^-25 of half a turn, 4 units of cos and sin, 2 more of sincospif itself;
    # the products by r, w, cos and sin and the pair's addition
    wide = (hd / 2 + 16) * U
    out_err = wide * _size(n * w, rot, interleaved)
    dy = _rotate(do, _turns(pos, freq, True), rot, interleaved)
    dn = dy * w
    dx = r * (dn - n * (dn * n).mean(-1, keepdim=True))
    s = _size(do, rot, interleaved)
    # r three times, and the sum of dn n, hd additions' roundings of its terms
    dx_err = (3 * hd + 64) * U * r * (s * w.abs() + n.abs() * (s * w.abs() * n.abs()).mean(-1, keepdim=True))
    return out, out_err, dx, dx_err, dy * n, s * n.abs()


CASES = [
    # T, hq, hk, hd, rot, interleaved, K, w dtype, ld beyond the heads, far
    (1, 1, 1, 16, 16, False, 1, BF, 0, False),
    (1, 32, 8, 128, 128, False, 1, BF, 1024, True),
    (2, 3, 1, 32, 16, True, 1, torch.float32, 0, False),
    (5, 5, 5, 48, 48, False, 2, BF, 8, True),
    (33, 4, 4, 64, 64, False, 3, BF, 0, False),
    (70, 10, 2, 80, 80, True, 3, torch.float32, 16, False),
    (70, 10, 2, 80, 32, False, 3, BF, 0, True),
    (257, 9, 3, 96, 48, True, 16, BF, 24, False),
    (131, 7, 1, 112, 112, False, 4, BF, 0, False),
    (300, 16, 2, 128, 64, True, 4, BF, 256, False),
    (64, 6, 6, 144, 144, False, 2, torch.float32, 0, False),
    (129, 3, 3, 192, 96, False, 2, BF, 0, True),
    (90, 8, 4, 256, 256, True, 3, BF, 0, False),
    (90, 2, 1, 256, 0, False, 3, BF, 8, False),
    (4097, 4, 2, 64, 32, False, 5, BF, 128, False),
    (3000, 40, 8, 128, 128, False, 7, BF, 0, False),
]


def _inputs(T, hq, hk, hd, rot, interleaved, K, wd, beyond, far):
    q, k, room = _fused(T, hq, hk, hd, 1, (hq + hk) * hd + beyond, std=2.0)
    w = [(1.0 + 0.3 * _normal(hd, seed=s)).to(wd) for s in (2, 3)]
    pos = torch.randint(-5, 1 << 22, (T,), generator=_gen(4), device=DEV) if far else torch.arange(T, device=DEV)
    freq = bk.rope_frequencies(rot, 1e4) if rot else []
    return q, k, room, w, pos, freq


@pytest.mark.parametrize("case", CASES)
def test_normed_and_rotated(case):
    T, hq, hk, hd, rot, interleaved, K, wd, beyond, far = case
    q, k, _, w, pos, freq = _inputs(*case)
    qo, ko, room = _fused(T, hq, hk, hd, 5, (hq + hk) * hd + beyond + 8)
    bk.bkmoo_qk_norm_forward(q, k, w[0], w[1], pos, freq, qo, ko, interleaved=interleaved)
    for x, o, wx in ((q, qo, w[0]), (k, ko, w[1])):
        ref, err, *_ = _reference(x, wx, torch.zeros_like(x), pos, freq, 1e-6, interleaved)
        assert bool(((o.double() - ref).abs() <= 1.01 * (err + 2.0 ** -8 * (ref.abs() + err))).all())
    assert bool((room[:, (hq + hk) * hd:] == 7.0).all())
    # int32 positions, and the results in the inputs' place: the same bits
    a, b = q.clone(), k.clone()
    bk.bkmoo_qk_norm_forward(a, b, w[0], w[1], pos.int(), list(freq), a, b, interleaved=interleaved)
    assert torch.equal(a, qo) and torch.equal(b, ko)


@pytest.mark.parametrize("accumulate,out", [(False, BF), (True, BF), (False, torch.float32), (True, torch.float32)])
@pytest.mark.parametrize("case", CASES)
def test_gradients_by_language(case, accumulate, out):
    T, hq, hk, hd, rot, interleaved, K, wd, beyond, far = case
    q, k, _, w, pos, freq = _inputs(*case)
    dqo, dko, _ = _fused(T, hq, hk, hd, 6, (hq + hk) * hd + beyond, std=0.1)
    dq, dk, room = _fused(T, hq, hk, hd, 7, (hq + hk) * hd + 16)
    rows = [T * i // K for i in range(K + 1)]
    if K > 2:
        rows[1] = 0
    start = 1 if T == 70 else 0                   # places at any element's address
    dw = [[_normal(hd + 1, seed=20 + i + 100 * s).to(out)[start:start + hd] for i in range(K)] for s in range(2)]
    before = [[g.double().clone() for g in side] for side in dw]

    def call(a, b, dq, dk, dw):
        bk.bkmoo_qk_norm_backward(a, b, q, k, w[0], w[1], pos, freq, rows, dq, dk, dw[0], dw[1], interleaved=interleaved,
                                  accumulate=accumulate)

    again = [[g.clone() for g in side] for side in dw]
    call(dqo, dko, dq, dk, dw)
    for s, (x, do, d, wx) in enumerate(((q, dqo, dq, w[0]), (k, dko, dk, w[1]))):
        _, _, ref, err, part, size = _reference(x, wx, do, pos, freq, 1e-6, interleaved)
        assert bool(((d.double() - ref).abs() <= 1.01 * (err + 2.0 ** -8 * (ref.abs() + err))).all())
        for i in range(K):
            a, b = rows[i], rows[i + 1]
            want, wide = part[a:b].sum((0, 1)), size[a:b].sum((0, 1)) * ((b - a) * x.shape[1] + hd / 2 + 24) * U
            if accumulate:
                want, wide = want + before[s][i], wide + U * before[s][i].abs()
            assert bool(((dw[s][i].double() - want).abs() <= 1.01 * (wide + HALF[out] * (want.abs() + wide))).all())
    assert bool((room[:, (hq + hk) * hd:] == 7.0).all())
    # in the place of dq_out and dk_out: the same bits
    a, b = dqo.clone(), dko.clone()
    call(a, b, a, b, again)
    assert torch.equal(a, dq) and torch.equal(b, dk)
    assert all(torch.equal(u, v) for s in range(2) for u, v in zip(dw[s], again[s]))
    # without the weights' gradients
    a, b = torch.empty_like(dqo), torch.empty_like(dko)
    bk.bkmoo_qk_norm_backward(dqo, dko, q, k, w[0], w[1], pos, freq, rows, a, b, interleaved=interleaved)
    assert torch.equal(a, dq) and torch.equal(b, dk)


def test_gradients_are_those_of_differences():
    """(f(x + h) - f(x - h)) / 2h of the forward formula in 64 bits, for some inputs."""
    T, hd, rot = 3, 32, 32
    x, w = _normal(T, 2, hd, seed=1).to(BF), (1.0 + 0.2 * _normal(hd, seed=2)).to(BF)
    do, pos, freq = _normal(T, 2, hd, seed=3).to(BF), torch.tensor([0, 9, 100], device=DEV), bk.rope_frequencies(rot, 100.0)
    d, dk = torch.empty_like(x), torch.empty_like(x)
    dw, dwk = torch.empty(hd, device=DEV), torch.empty(hd, device=DEV)
    bk.bkmoo_qk_norm_backward(do, do, x, x, w, w, pos, freq, [0, T], d, dk, [dw], [dwk])
    assert torch.equal(d, dk) and torch.equal(dw, dwk)

    def f(x, w):
        y = x / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w
        return float((_rotate(y, _turns(pos, freq, False), rot, False) * do.double()).sum())

    h = 1e-4
    for t, head, c in ((0, 0, 0), (1, 1, 31), (2, 0, 17)):
        hi, lo = x.double(), x.double()
        hi[t, head, c] += h
        lo[t, head, c] -= h
        diff = (f(hi, w.double()) - f(lo, w.double())) / (2 * h)
        # h^2 of a third derivative that is a few times 1, fp64's rounding over h, and bf16's
        assert abs(float(d[t, head, c]) - diff) <= 2.0 ** -8 * abs(diff) + 2e-6
    for c in (0, 20):
        hi, lo = w.double(), w.double()
        hi[c] += h
        lo[c] -= h
        diff = (f(x.double(), hi) - f(x.double(), lo)) / (2 * h)
        assert abs(float(dw[c]) - diff) <= 2e-5


def test_far_positions_keep_their_angle():
    """Position 2^40 - 1 is as exact as position 3."""
    T, hd = 4, 64
    pos = torch.tensor([3, 2 ** 40 - 1, -(2 ** 40), 2 ** 31 + 5], device=DEV)
    x = _normal(T, 1, hd, seed=1).to(BF)
    o, o2 = torch.empty_like(x), torch.empty_like(x)
    # frequencies that are whole 4096ths of a turn: the angles are known at any position
    freq = [2 * math.pi * (i + 1) / 4096.0 for i in range(hd // 2)]
    one = torch.ones(hd, device=DEV)
    bk.bkmoo_qk_norm_forward(x, x, one, one, pos, freq, o, o2)
    i = torch.arange(1, hd // 2 + 1, device=DEV)
    a = ((pos[:, None] % 4096) * i % 4096).double() * (2 * math.pi / 4096)
    # the frequency's own roundings and those into turns, four of 2^-53 of at most 1/20 radian, over
    # 2^40 positions
    y = x.double() / torch.sqrt(x.double().square().mean(-1, keepdim=True) + 1e-6)
    turn = torch.polar(torch.ones_like(a), a)[:, None]
    ref, s = _rotate(y, turn, hd, False), _size(y, hd, False)
    err = (hd / 2 + 16) * U * s + 2.0 ** -15 * s
    assert bool(((o.double() - ref).abs() <= 1.01 * (err + 2.0 ** -8 * (ref.abs() + err))).all())


def test_no_rows_and_heads_of_zeros():
    hd, freq = 64, bk.rope_frequencies(64, 1e4)
    w = torch.ones(hd, device=DEV)
    q, k, _ = _fused(0, 2, 1, hd, 1)
    pos = torch.empty(0, dtype=torch.int64, device=DEV)
    bk.bkmoo_qk_norm_forward(q, k, w, w, pos, freq, q.clone(), k.clone())
    dw = [[torch.ones(hd, device=DEV) for _ in range(2)] for _ in range(2)]
    bk.bkmoo_qk_norm_backward(q, k, q, k, w, w, pos, freq, [0, 0, 0], q.clone(), k.clone(), dw[0], dw[1], accumulate=True)
    assert all(bool((g == 1).all()) for side in dw for g in side)
    bk.bkmoo_qk_norm_backward(q, k, q, k, w, w, pos, freq, [0, 0, 0], q.clone(), k.clone(), dw[0], dw[1])
    assert all(bool((g == 0).all()) for side in dw for g in side)
    # heads of zeros: 0, and a gradient of r dy w
    x = torch.zeros(6, 3, hd, dtype=BF, device=DEV)
    do = _normal(6, 3, hd, seed=2).to(BF)
    o, d, d2 = (torch.empty_like(x) for _ in range(3))
    pos = torch.zeros(6, dtype=torch.int64, device=DEV)
    bk.bkmoo_qk_norm_forward(x, x, w, w, pos, freq, o, d, eps=1e-4)
    assert bool((o == 0).all()) and bool((d == 0).all())
    bk.bkmoo_qk_norm_backward(do, do, x, x, w, w, pos, freq, [0, 6], d, d2, [dw[0][0]], [dw[0][1]], eps=1e-4)
    assert bool(((d.double() - 100 * do.double()).abs() <= 2.0 ** -8 * 1.01 * (100 * do.double()).abs()).all())
    assert bool((dw[0][0] == 0).all())


def test_a_head_keeps_its_nan():
    T, h, hd = 40, 3, 96
    freq, pos, w = bk.rope_frequencies(hd, 1e4), torch.arange(T, device=DEV), torch.ones(hd, dtype=BF, device=DEV)
    x, do = _normal(T, h, hd, seed=1).to(BF), _normal(T, h, hd, seed=2).to(BF)
    x[7, 1, 3] = math.nan
    o, o2, d, d2 = (torch.empty_like(x) for _ in range(4))
    dw = [[torch.empty(hd, device=DEV) for _ in range(2)] for _ in range(2)]
    bk.bkmoo_qk_norm_forward(x, x, w, w, pos, freq, o, o2)
    bk.bkmoo_qk_norm_backward(do, do, x, x, w, w, pos, freq, [0, 20, T], d, d2, dw[0], dw[1])
    for t in (o, o2, d, d2):
        bad = torch.isnan(t)
        assert bool(bad[7, 1].all()) and int(bad.sum()) == hd
    assert bool(torch.isnan(dw[0][0]).all()) and not bool(torch.isnan(dw[0][1]).any())


def test_tokens_beyond_32_bits():
    """Strides that put the last tokens past 2^32 elements."""
    T, h, hd, ld = 9, 2, 64, 1 << 29
    room = torch.empty((T - 1) * ld + 4 * h * hd, dtype=BF, device=DEV)
    q, k = (torch.as_strided(room, (T, h, hd), (ld, hd, 1), s * h * hd) for s in range(2))
    qo, ko = (torch.as_strided(room, (T, h, hd), (ld, hd, 1), s * h * hd) for s in (2, 3))
    for s, x in enumerate((q, k)):
        x.copy_(_normal(T, h, hd, seed=s))
    w, pos, freq = torch.ones(hd, device=DEV), torch.arange(T, device=DEV), bk.rope_frequencies(hd, 1e4)
    bk.bkmoo_qk_norm_forward(q, k, w, w, pos, freq, qo, ko)
    a, b = torch.empty(T, h, hd, dtype=BF, device=DEV), torch.empty(T, h, hd, dtype=BF, device=DEV)
    bk.bkmoo_qk_norm_forward(q.contiguous(), k.contiguous(), w, w, pos, freq, a, b)
    assert torch.equal(qo, a) and torch.equal(ko, b)
    bk.bkmoo_qk_norm_backward(a, b, q.contiguous(), k.contiguous(), w, w, pos, freq, [0, T], a, b)
    bk.bkmoo_qk_norm_backward(qo, ko, q, k, w, w, pos, freq, [0, T], qo, ko)
    assert torch.equal(qo, a) and torch.equal(ko, b)


def test_captured_and_replayed_and_on_another_stream():
    case = (700, 8, 2, 128, 128, False, 3, BF, 0, False)
    T, hq, hk, hd = case[:4]
    q, k, room, w, pos, freq = _inputs(*case)
    dqo, dko, _ = _fused(T, hq, hk, hd, 6)
    rows = [0, 100, 450, T]
    qo, ko, dq, dk = (torch.empty_like(t) for t in (q, k, q, k))
    dw = [[torch.empty(hd, device=DEV) for _ in range(3)] for _ in range(2)]

    def step(stream=None):
        bk.bkmoo_qk_norm_forward(q, k, w[0], w[1], pos, freq, qo, ko, stream=stream)
        bk.bkmoo_qk_norm_backward(dqo, dko, q, k, w[0], w[1], pos, freq, rows, dq, dk, dw[0], dw[1], stream=stream)

    outs = [qo, ko, dq, dk] + dw[0] + dw[1]
    step()
    want = [t.clone() for t in outs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for t in outs:
            t.zero_()
    step(side)
    side.synchronize()
    assert all(torch.equal(u, v) for u, v in zip(want, outs))
    # a replay takes the inputs of its time; the frequencies are those of the capture
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    pos += 1000
    room[:, :(hq + hk) * hd] = _normal(T, (hq + hk) * hd, seed=40)
    g.replay()
    got = [t.clone() for t in outs]
    step()
    assert all(torch.equal(u, v) for u, v in zip(got, outs))
