"""The embedding and its gradient apart by language against the formula in 64 bits, on the
GPU."""
import math

import pytest
import torch

from paper_2606_05613_gb300 import native as bk

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24                                   # a rounding to fp32, relative
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _matrix(rows, cols, dtype, seed, ld=None, ahead=0):
    """A matrix of normal numbers in rows of `ld`, the first `ahead` elements into its memory;
    the memory between the rows holds 7."""
    ld = cols if ld is None else ld
    room = torch.full((ahead + max(rows, 1) * ld,), 7.0, dtype=dtype, device=DEV)
    m = room[ahead:].view(max(rows, 1), ld)[:rows, :cols]
    m.copy_(torch.randn(rows, cols, generator=_gen(seed), device=DEV))
    return m, room


def _ids(T, V, seed, dtype=torch.int64, distinct=None):
    n = V if distinct is None else distinct
    ids = torch.randint(0, n, (T,), generator=_gen(seed), device=DEV)
    if T > 3:
        ids[1], ids[T // 2], ids[T - 1] = -1, V, -100      # padding
    return ids.to(dtype)


def _forward_is_right(table, ids, y, scale):
    V = table.shape[0]
    ok = (ids >= 0) & (ids < V)
    ref = table.double()[ids.long().clamp(0, V - 1)] * scale * ok[:, None]
    # the scale and the product in fp32, and the result's rounding
    assert bool(((y.double() - ref).abs() <= ref.abs() * (2 * U + HALF[table.dtype]) * 1.01).all())


@pytest.mark.parametrize("id_type", [torch.int64, torch.int32])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,V,D,ld,ahead,scale", [
    (1, 1, 1, 1, 0, 1.0), (1, 7, 8, 8, 0, 0.5), (2, 5, 9, 9, 0, 1.0), (33, 100, 64, 64, 0, 8.0),
    (33, 100, 64, 72, 0, 8.0), (33, 100, 64, 65, 0, 8.0), (33, 100, 64, 64, 1, 8.0), (257, 1001, 771, 771, 0, 0.3),
    (1500, 501, 2048, 2048, 8, math.sqrt(2048)), (40, 90, 12, 16, 0, -2.0), (5, 50, 8192, 8200, 0, 0.0)])
def test_rows_by_token(T, V, D, ld, ahead, scale, dtype, id_type):
    table, _ = _matrix(V, D, dtype, 1, ld, ahead)
    ids = _ids(T, V, 2, id_type)
    y, room = _matrix(T, D, dtype, 3, ld, ahead)
    bk.bkmoo_embedding_forward(table, ids, y, scale=scale)
    _forward_is_right(table, ids, y, scale)
    assert int((room == 7.0).sum()) >= room.numel() - T * D       # nothing between the rows


def test_padding_reads_nothing():
    """Rows of padding are 0 whatever the table holds."""
    table = torch.full((4, 64), math.nan, device=DEV)
    ids = torch.tensor([-1, 4, 1 << 40, -(1 << 40)], device=DEV)
    y = torch.ones(4, 64, device=DEV)
    bk.bkmoo_embedding_forward(table, ids, y, scale=3.0)
    assert bool((y == 0).all())


def _bounds(T, K, empty):
    rows = [T * k // K for k in range(K + 1)]
    if empty and K > 1:
        rows[1] = rows[0]
    return rows


def _gradient_is_right(dy, ids, rows, dw, scale, before=None):
    V, D = dw[0].shape
    for k, (i, j) in enumerate(zip(rows, rows[1:])):
        ok = ((ids[i:j] >= 0) & (ids[i:j] < V)).nonzero()[:, 0] + i
        at = ids[ok].long()
        total, size = (torch.zeros(V, D, dtype=torch.float64, device=DEV) for _ in range(2))
        total.index_add_(0, at, dy[ok].double())
        size.index_add_(0, at, dy[ok].double().abs())
        n = torch.bincount(at, minlength=V)[:, None]
        ref, size = total * scale, size * abs(scale)
        if before is not None:
            ref, size = ref + before[k].double(), size + before[k].double().abs()
        # n additions, the scale and its product (or one fused addition), the rounding
        bound = (n + 2) * U * size + HALF[dw[k].dtype] * (ref.abs() + (n + 2) * U * size)
        bound[n[:, 0] == 0] = 0
        assert bool(((dw[k].double() - ref).abs() <= bound * 1.01).all())


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("dtype,out", [(torch.bfloat16, torch.bfloat16), (torch.float32, torch.float32),
                                       (torch.bfloat16, torch.float32), (torch.float32, torch.bfloat16)])
@pytest.mark.parametrize("T,V,D,K,distinct,ld,ahead", [
    (1, 1, 1, 1, 1, 1, 0), (1, 9, 8, 1, 9, 8, 0), (31, 9, 16, 2, 9, 16, 0), (32, 3, 24, 1, 1, 24, 0),
    (33, 3, 24, 1, 1, 24, 0), (65, 40, 256, 3, 2, 264, 0), (100, 1000, 257, 4, 60, 257, 0),
    (1024, 5000, 40, 16, 30, 40, 0), (1025, 50, 264, 3, 50, 264, 8), (1500, 700, 129, 3, 3, 131, 1),
    (5000, 20000, 64, 4, 20000, 64, 0), (33000, 300, 12, 2, 300, 12, 0), (40000, 1 << 20, 8, 3, 1 << 20, 8, 0)])
def test_gradients_by_token_and_language(T, V, D, K, distinct, ld, ahead, dtype, out, accumulate):
    dy, _ = _matrix(T, D, dtype, 5, ld, ahead)
    ids = _ids(T, V, 6, torch.int32 if D % 16 else torch.int64, distinct)
    rows = _bounds(T, K, T % 3 == 0)
    rooms = [torch.randn(V * D + 1, generator=_gen(7 + k), device=DEV).to(out) for k in range(K)]
    start = 1 if T == 1500 else 0                 # places at any element's address
    dw = [r[start:start + V * D].view(V, D) for r in rooms]
    before = [w.clone() for w in dw] if accumulate else None
    scale = 0.5 if D == 40 else math.sqrt(D)
    bk.bkmoo_embedding_backward(dy, ids, rows, dw, scale=scale, accumulate=accumulate)
    first = [w.clone() for w in dw]
    _gradient_is_right(dy, ids, rows, dw, scale, before)
    # the same call gives the same bits
    if accumulate:
        for w, b in zip(dw, before):
            w.copy_(b)
    bk.bkmoo_embedding_backward(dy, ids, rows, dw, scale=scale, accumulate=accumulate)
    assert all(torch.equal(u, v) for u, v in zip(first, dw))


def test_one_token_in_every_row():
    """A sum over all rows of a language, joined over many pieces."""
    T, V, D = 70000, 11, 264
    dy, _ = _matrix(T, D, torch.bfloat16, 8)
    ids = torch.full((T,), 5, device=DEV)
    rows = [0, 29999, 30000, T]
    dw = [torch.randn(V, D, device=DEV) for _ in range(3)]
    before = [w.clone() for w in dw]
    bk.bkmoo_embedding_backward(dy, ids, rows, dw, scale=0.25, accumulate=True)
    _gradient_is_right(dy, ids, rows, dw, 0.25, before)


def test_padding_has_no_gradient():
    T, V, D = 300, 10, 64
    dy = torch.full((T, D), math.nan, dtype=torch.bfloat16, device=DEV)
    ids = torch.full((T,), -1, device=DEV)
    ids[150:] = V
    dw = [torch.ones(V, D, device=DEV) for _ in range(2)]
    bk.bkmoo_embedding_backward(dy, ids, [0, 100, T], dw, accumulate=True)
    assert all(bool((w == 1).all()) for w in dw)
    bk.bkmoo_embedding_backward(dy, ids, [0, 100, T], dw)
    assert all(bool((w == 0).all()) for w in dw)


def test_no_rows():
    dw = [torch.ones(4, 8, device=DEV) for _ in range(2)]
    dy, ids = torch.empty(0, 8, device=DEV), torch.empty(0, dtype=torch.int64, device=DEV)
    y = torch.empty(0, 8, device=DEV)
    bk.bkmoo_embedding_forward(dw[0], ids, y)
    bk.bkmoo_embedding_backward(dy, ids, [0, 0, 0], dw, accumulate=True)
    assert all(bool((w == 1).all()) for w in dw)
    bk.bkmoo_embedding_backward(dy, ids, [0, 0, 0], dw)
    assert all(bool((w == 0).all()) for w in dw)


def test_a_language_keeps_its_nan():
    T, V, D, rows = 200, 30, 64, [0, 90, 200]
    dy, _ = _matrix(T, D, torch.float32, 9)
    dy[50] = math.nan
    ids = _ids(T, V, 10)
    dw = [torch.empty(V, D, device=DEV) for _ in range(2)]
    bk.bkmoo_embedding_backward(dy, ids, rows, dw)
    assert bool(torch.isnan(dw[0][ids[50]]).all()) and int(torch.isnan(dw[0]).sum()) == D
    assert not bool(torch.isnan(dw[1]).any())


def test_places_beyond_32_bits():
    """Rows of a table and of a gradient past 2^32 elements."""
    V, D = 70001, 65536
    table = torch.empty(V, D, dtype=torch.bfloat16, device=DEV)
    ids = torch.tensor([0, V - 1, 65537, V, V - 1, 40000], device=DEV)
    for v in (0, V - 1, 65537, 40000):
        table[v].copy_(torch.randn(D, generator=_gen(v), device=DEV))
    y = torch.empty(6, D, dtype=torch.bfloat16, device=DEV)
    bk.bkmoo_embedding_forward(table, ids, y, scale=2.0)
    for t, v in enumerate(ids.tolist()):
        assert torch.equal(y[t], table[v] * 2 if v < V else torch.zeros_like(y[t]))
    dy, _ = _matrix(6, D, torch.bfloat16, 11)
    before = table.clone()
    bk.bkmoo_embedding_backward(dy, ids, [0, 6], [table], accumulate=True)
    for v, rows in ((0, [0]), (V - 1, [1, 4]), (65537, [2]), (40000, [5])):
        ref = before[v].double() + dy[rows].double().sum(0)
        size = before[v].double().abs() + dy[rows].double().abs().sum(0)
        assert bool(((table[v].double() - ref).abs() <= 1.01 * (4 * U * size + 2.0 ** -8 * (ref.abs() + 4 * U * size))).all())
    for v in (1, 65536, 65538, V - 2):
        assert torch.equal(table[v].view(torch.int16), before[v].view(torch.int16))


def test_captured_and_replayed_and_on_another_stream():
    T, V, D, rows = 1100, 300, 136, [0, 400, 1100]
    table, _ = _matrix(V, D, torch.bfloat16, 12)
    dy, _ = _matrix(T, D, torch.bfloat16, 13)
    ids = _ids(T, V, 14)
    y = torch.empty(T, D, dtype=torch.bfloat16, device=DEV)
    dw = [torch.empty(V, D, dtype=torch.bfloat16, device=DEV) for _ in range(2)]

    def step(stream=None):
        bk.bkmoo_embedding_forward(table, ids, y, scale=3.0, stream=stream)
        bk.bkmoo_embedding_backward(dy, ids, rows, dw, scale=3.0, stream=stream)

    step()
    want = [y.clone()] + [w.clone() for w in dw]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y.zero_(), dw[0].zero_(), dw[1].zero_()
    step(side)
    side.synchronize()
    assert all(torch.equal(u, v) for u, v in zip(want, [y] + dw))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for shift in (0, 17):
        ids.copy_(_ids(T, V, 14 + shift))
        g.replay()
        _forward_is_right(table, ids, y, 3.0)
        _gradient_is_right(dy, ids, rows, dw, 3.0)
