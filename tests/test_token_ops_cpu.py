"""CPU: the entry points of the embedding, the norms of queries and keys and the token log
probabilities refuse bad arguments before they touch a GPU.  Addresses are made up and
never read."""
import ctypes
import math
import os
import re

import pytest
import torch

from paper_2606_05613_gb300 import build as nb
from paper_2606_05613_gb300 import native as bk
from test_binding_cpu import _T, called      # noqa: F401 (a fixture)

OK, INVALID, WS = bk.BKMOO_OK, bk.BKMOO_ERR_INVALID, bk.BKMOO_ERR_WORKSPACE
P = 1 << 40                       # an aligned address
INF, NAN = math.inf, math.nan


@pytest.fixture(scope="module", autouse=True)
def _built():
    nb.build()
    bk.load()


def _rows(*r):
    return (ctypes.c_int64 * len(r))(*r)


def _ptrs(*p):
    return (ctypes.c_void_p * len(p))(*p)


def _freq(*f):
    return (ctypes.c_double * len(f))(*f)


def _call(fn, args, changes):
    a = dict(args)
    assert set(changes) <= set(a)
    a.update(changes)
    return fn(*a.values())


LOOKUP = dict(table=P, ld=64, dt=1, V=100, D=64, ids=P, nb=8, T=5, scale=1.0, y=P, ldy=64, stream=None)


@pytest.mark.parametrize("bad", [dict(table=None), dict(table=P + 1), dict(dt=0, table=P + 2), dict(ld=63), dict(ldy=63),
                                 dict(dt=2), dict(dt=-1), dict(V=0), dict(V=1 << 28), dict(D=0), dict(D=(1 << 23) + 1),
                                 dict(ids=None), dict(ids=P + 4), dict(nb=2), dict(nb=4, ids=P + 2), dict(T=-1), dict(T=1 << 31),
                                 dict(scale=INF), dict(scale=NAN), dict(scale=1e39), dict(y=None), dict(y=P + 1), dict(ld=1 << 39)])
def test_embedding_forward_refuses(bad):
    assert _call(bk.load().bkmoo_embedding_forward, LOOKUP, bad) == INVALID


def test_embedding_forward_without_rows_does_nothing():
    assert _call(bk.load().bkmoo_embedding_forward, LOOKUP, dict(T=0, ids=None, y=None)) == OK


SUMS = dict(dy=P, ld=64, dt=1, ids=P, nb=8, T=5, V=100, D=64, scale=1.0, K=2, rows=_rows(0, 2, 5), dw=_ptrs(P, P + (1 << 30)), wt=1, acc=0,
            ws=P, size=1 << 40, stream=None)


@pytest.mark.parametrize("bad", [dict(dy=None), dict(dy=P + 1), dict(dt=0, dy=P + 2), dict(ld=63), dict(dt=2), dict(wt=2),
                                 dict(ids=None), dict(ids=P + 4), dict(nb=1), dict(T=-1), dict(T=1 << 31), dict(V=0),
                                 dict(V=1 << 28), dict(D=0), dict(scale=NAN), dict(scale=-1e39), dict(K=0), dict(K=17),
                                 dict(rows=None), dict(rows=_rows(0, 2, 4)), dict(rows=_rows(0, 6, 5)), dict(rows=_rows(1, 2, 5)),
                                 dict(dw=None), dict(dw=_ptrs(P, None)), dict(dw=_ptrs(P, P + 1)), dict(wt=0, dw=_ptrs(P + 2, P)),
                                 dict(ws=None), dict(ws=P + 128), dict(V=1 << 20, D=1 << 20, ld=1 << 20)])
def test_embedding_backward_refuses(bad):
    assert _call(bk.load().bkmoo_embedding_backward, SUMS, bad) == INVALID


def test_gradients_that_overlap_are_refused():
    """Two languages that add to one place would lose each other's sums."""
    fn, grads = bk.load().bkmoo_embedding_backward, lambda d: dict(dw=_ptrs(P, P + d), size=0)
    assert _call(fn, SUMS, grads(0)) == INVALID and _call(fn, SUMS, grads(100 * 64 * 2 - 2)) == INVALID
    assert _call(fn, SUMS, grads(100 * 64 * 2)) == WS and _call(fn, SUMS, dict(wt=0, **grads(100 * 64 * 2))) == INVALID
    fn = bk.load().bkmoo_qk_norm_backward
    for q, k in (((P, P), (P + 256, P + 512)), ((P, P + 256), (P + 512, P + 126)), ((P, P + 256), (P, P + 512))):
        assert _call(fn, BACK, dict(dwq=_ptrs(*q), dwk=_ptrs(*k), size=0)) == INVALID
    assert _call(fn, BACK, dict(size=0)) == WS


def test_embedding_backward_needs_its_workspace():
    for T, D in ((5, 64), (1025, 300)):
        n = bk.bkmoo_embedding_backward_workspace_size(T, D)
        assert n > 0 and _call(bk.load().bkmoo_embedding_backward, SUMS,
                               dict(T=T, D=D, ld=D, rows=_rows(0, 2, T), size=n - 1)) == WS
    assert bk.bkmoo_embedding_backward_workspace_size(0, 8) == 0
    for T, D in ((-1, 8), (4, 0), (1 << 31, 8)):
        with pytest.raises(bk.BkmooError):
            bk.bkmoo_embedding_backward_workspace_size(T, D)
    assert bk.load().bkmoo_embedding_backward_workspace_size(4, 8, None) == INVALID
    # added to, no rows: nothing is touched
    assert _call(bk.load().bkmoo_embedding_backward, SUMS,
                 dict(T=0, rows=_rows(0, 0, 0), dy=None, ids=None, acc=1, ws=None, size=0)) == OK


NORM = dict(q=P, ldq=512, k=P, ldk=512, wq=P, wk=P, wt=1, T=5, hq=4, hk=2, hd=64, pos=P, nb=8, freq=_freq(*[0.5] * 32), rot=64,
            inter=0, eps=1e-6, qo=P + (1 << 30), ldqo=512, ko=P + (1 << 30), ldko=512, stream=None)
BAD_NORM = [dict(q=None), dict(q=P + 8), dict(k=None), dict(k=P + 2), dict(ldq=248), dict(ldq=516), dict(ldk=124), dict(wq=None),
            dict(wk=None), dict(wq=P + 1), dict(wt=0, wk=P + 2), dict(wt=2), dict(T=-1), dict(T=1 << 31), dict(hq=0), dict(hk=0),
            dict(hq=1 << 17, ldq=1 << 24), dict(hd=8, rot=0), dict(hd=72), dict(hd=272, rot=64, ldq=1088, ldk=1088), dict(pos=None),
            dict(pos=P + 4), dict(nb=3), dict(freq=None), dict(rot=8), dict(rot=80), dict(rot=-16), dict(eps=-1.0), dict(eps=NAN),
            dict(eps=INF), dict(freq=_freq(*[0.5] * 31 + [INF])), dict(freq=_freq(*[NAN] + [0.5] * 31))]


@pytest.mark.parametrize("bad", BAD_NORM + [dict(qo=None), dict(ko=None), dict(qo=P + 4), dict(ldqo=248), dict(ldko=132),
                                            dict(qo=P, ldqo=520), dict(ko=P, ldko=520)])
def test_qk_norm_forward_refuses(bad):
    assert _call(bk.load().bkmoo_qk_norm_forward, NORM, bad) == INVALID


def test_qk_norm_forward_without_rows_does_nothing():
    assert _call(bk.load().bkmoo_qk_norm_forward, NORM, dict(T=0, q=None, k=None, qo=None, ko=None, pos=None)) == OK


BACK = dict(dqo=P, ld1=512, dko=P, ld2=512, q=P, ldq=512, k=P, ldk=512, wq=P, wk=P, wt=1, T=5, hq=4, hk=2, hd=64, pos=P, nb=8,
            freq=_freq(*[0.5] * 32), rot=64, inter=0, eps=1e-6, K=2, rows=_rows(0, 2, 5), dq=P + (1 << 30), ld3=512,
            dk=P + (1 << 30), ld4=512, dwq=_ptrs(P, P + 128), dwk=_ptrs(P + 256, P + 384), dt=1, acc=0, ws=P, size=1 << 40, stream=None)


@pytest.mark.parametrize("bad", BAD_NORM + [dict(dqo=None), dict(dko=P + 8), dict(ld1=248), dict(ld2=516), dict(dq=None),
                                            dict(dk=P + 8), dict(ld3=248), dict(ld4=4), dict(dq=P, ld3=520), dict(dk=P, ld4=520),
                                            dict(K=0), dict(K=17), dict(rows=None), dict(rows=_rows(0, 2, 4)),
                                            dict(rows=_rows(0, 6, 5)), dict(dwq=None), dict(dwk=None), dict(dwq=_ptrs(P, None)),
                                            dict(dwk=_ptrs(P, P + 1)), dict(dt=0, dwk=_ptrs(P, P + 2)), dict(dt=2), dict(ws=None),
                                            dict(ws=P + 64)])
def test_qk_norm_backward_refuses(bad):
    assert _call(bk.load().bkmoo_qk_norm_backward, BACK, bad) == INVALID


def test_qk_norm_backward_needs_its_workspace():
    n = bk.bkmoo_qk_norm_backward_workspace_size(64)
    assert n > 0 and _call(bk.load().bkmoo_qk_norm_backward, BACK, dict(size=n - 1)) == WS
    for width in (0, 8, 72, 272):
        with pytest.raises(bk.BkmooError):
            bk.bkmoo_qk_norm_backward_workspace_size(width)
    assert bk.load().bkmoo_qk_norm_backward_workspace_size(64, None) == INVALID
    none = dict(T=0, rows=_rows(0, 0, 0), dqo=None, dko=None, q=None, k=None, dq=None, dk=None, pos=None)
    assert _call(bk.load().bkmoo_qk_norm_backward, BACK, dict(none, dwq=None, dwk=None, ws=None, size=0)) == OK
    assert _call(bk.load().bkmoo_qk_norm_backward, BACK, dict(none, acc=1)) == OK


LOGP = dict(z=P, ld=100, dt=1, T=5, V=100, targets=P, nb=8, logp=P, stats=P, entropy=P, n=3, ids=P, top=P, stream=None)


@pytest.mark.parametrize("bad", [dict(z=None), dict(z=P + 1), dict(dt=0, z=P + 2), dict(ld=99), dict(ld=1 << 39), dict(dt=2),
                                 dict(T=-1), dict(T=1 << 31), dict(V=0), dict(V=(1 << 30) + 1, ld=1 << 31), dict(targets=None),
                                 dict(targets=P + 4), dict(nb=0), dict(logp=None), dict(logp=P + 2), dict(stats=P + 4),
                                 dict(entropy=P + 2), dict(n=-1), dict(n=33), dict(V=2, n=3), dict(ids=None), dict(ids=P + 4),
                                 dict(top=None), dict(top=P + 2)])
def test_token_logp_forward_refuses(bad):
    assert _call(bk.load().bkmoo_token_logp_forward, LOGP, bad) == INVALID


GRAD = dict(z=P, ld=100, dt=1, T=5, V=100, targets=P, nb=8, stats=P, entropy=P, g=P, h=P, dz=P + (1 << 30), ldd=100, stream=None)


@pytest.mark.parametrize("bad", [dict(z=None), dict(z=P + 1), dict(ld=99), dict(dt=3), dict(T=-1), dict(V=0), dict(targets=None),
                                 dict(targets=P + 1), dict(nb=16), dict(stats=None), dict(stats=P + 4), dict(entropy=None),
                                 dict(g=None), dict(g=P + 2), dict(h=P + 2), dict(dz=None), dict(dz=P + 1), dict(ldd=99),
                                 dict(dz=P, ldd=104), dict(T=(1 << 31) - 1024, V=1 << 30, ld=1 << 30, ldd=1 << 30)])
def test_token_logp_backward_refuses(bad):
    assert _call(bk.load().bkmoo_token_logp_backward, GRAD, bad) == INVALID


def test_token_logp_without_rows_does_nothing():
    assert _call(bk.load().bkmoo_token_logp_forward, LOGP, dict(T=0, z=None, targets=None, logp=None, stats=None)) == OK
    assert _call(bk.load().bkmoo_token_logp_backward, GRAD, dict(T=0, z=None, targets=None, stats=None, g=None, dz=None)) == OK


B, F, I, I32 = torch.bfloat16, torch.float32, torch.int64, torch.int32


def test_binding_takes_what_it_should(called):      # noqa: F811
    bk.bkmoo_embedding_forward(_T(9, 7), _T(4, dtype=I), _T(4, 7))
    bk.bkmoo_embedding_backward(_T(4, 7), _T(4, dtype=I32), [0, 1, 4], [_T(9, 7, dtype=F)] * 2, ws=_T(1 << 20, dtype=torch.uint8))
    assert [c[:15] for c in called] == ["bkmoo_embedding"] * 2


@pytest.mark.parametrize("bad", [
    lambda: bk.bkmoo_embedding_forward(_T(9, 8), _T(4, dtype=F), _T(4, 8)),
    lambda: bk.bkmoo_embedding_forward(_T(9, 8), _T(4, dtype=I, dev=1), _T(4, 8)),
    lambda: bk.bkmoo_embedding_forward(_T(9, 8), _T(4, dtype=I), _T(5, 8)),
    lambda: bk.bkmoo_embedding_forward(_T(9, 8), _T(4, dtype=I), _T(4, 8, dtype=F)),
    lambda: bk.bkmoo_embedding_forward(_T(9, 8), _T(4, dtype=I, contiguous=False), _T(4, 8)),
    lambda: bk.bkmoo_embedding_forward(_T(9, 8, dev=-1), _T(4, dtype=I), _T(4, 8)),
    lambda: bk.bkmoo_embedding_backward(_T(4, 8), _T(4, dtype=I), [0, 4], [_T(9, 7)]),
    lambda: bk.bkmoo_embedding_backward(_T(4, 8), _T(4, dtype=I), [0, 4], []),
    lambda: bk.bkmoo_embedding_backward(_T(4, 8), _T(4, dtype=I), [0, 4], [_T(9, 8), _T(9, 8)]),
    lambda: bk.bkmoo_embedding_backward(_T(4, 8), _T(4, dtype=I), [0, 3], [_T(9, 8)]),
    lambda: bk.bkmoo_embedding_backward(_T(4, 8), _T(5, dtype=I), [0, 4], [_T(9, 8)]),
    lambda: bk.bkmoo_embedding_backward(_T(4, 8), _T(4, dtype=I), [0, 4], [_T(9, 8)], ws=_T(1 << 20, dtype=torch.uint8, dev=-1)),
    lambda: bk.bkmoo_token_logp_forward(_T(4, 8), _T(4, dtype=I), _T(4)),
    lambda: bk.bkmoo_token_logp_forward(_T(4, 8), _T(3, dtype=I), _T(4, dtype=F)),
    lambda: bk.bkmoo_token_logp_forward(_T(4, 8), _T(4, dtype=I), _T(4, dtype=F), stats=_T(4, dtype=F)),
    lambda: bk.bkmoo_token_logp_forward(_T(4, 8), _T(4, dtype=I), _T(4, dtype=F), top_ids=_T(4, 2, dtype=I)),
    lambda: bk.bkmoo_token_logp_forward(_T(4, 8), _T(4, dtype=I), _T(4, dtype=F), None, None, _T(4, 2, dtype=I), _T(4, 3, dtype=F)),
    lambda: bk.bkmoo_token_logp_forward(_T(4, 8), _T(4, dtype=I), _T(4, dtype=F), None, None, _T(4, 2, dtype=I32), _T(4, 2, dtype=F)),
    lambda: bk.bkmoo_token_logp_backward(_T(4, 8), _T(4, dtype=I), _T(8, dtype=F), _T(4, dtype=F), _T(4, 9)),
    lambda: bk.bkmoo_token_logp_backward(_T(4, 8), _T(4, dtype=I), _T(8, dtype=F), _T(4, dtype=F), _T(4, 8, dtype=F)),
    lambda: bk.bkmoo_token_logp_backward(_T(4, 8), _T(4, dtype=I), _T(8, dtype=F), _T(4, dtype=F), _T(4, 8), None, _T(4, dtype=F)),
])
def test_binding_refuses(called, bad):              # noqa: F811
    with pytest.raises(ValueError):
        bad()
    assert called == []


class _H(_T):
    """[tokens, heads, width]."""

    def stride(self):
        return (self.shape[1] * self.shape[2], self.shape[2], 1)


def _norm(**changes):
    a = dict(q=_H(5, 4, 64), k=_H(5, 2, 64), w_q=_T(64), w_k=_T(64), positions=_T(5, dtype=I), inv_freq=[0.5] * 32,
             q_out=_H(5, 4, 64), k_out=_H(5, 2, 64))
    a.update(changes)
    bk.bkmoo_qk_norm_forward(**a)


def _norm_back(**changes):
    a = dict(dq_out=_H(5, 4, 64), dk_out=_H(5, 2, 64), q=_H(5, 4, 64), k=_H(5, 2, 64), w_q=_T(64), w_k=_T(64),
             positions=_T(5, dtype=I), inv_freq=[0.5] * 32, rows=[0, 5], dq=_H(5, 4, 64), dk=_H(5, 2, 64), dw_q=[_T(64)],
             dw_k=[_T(64)], ws=_T(1 << 20, dtype=torch.uint8))
    a.update(changes)
    bk.bkmoo_qk_norm_backward(**a)


COMMON = [dict(q=_H(5, 4, 64, dev=-1)), dict(q=_H(5, 4, 64, dtype=F)), dict(k=_H(4, 2, 64)), dict(k=_H(5, 2, 32)),
          dict(w_q=_T(32)), dict(w_k=_T(64, dtype=F)), dict(w_q=_T(64, dev=1)), dict(positions=_T(4, dtype=I)),
          dict(positions=_T(5, dtype=F))]


def test_qk_norm_binding_refuses(called):           # noqa: F811
    _norm()
    _norm_back()
    assert len(called) == 2
    for bad in COMMON + [dict(q_out=_H(5, 3, 64)), dict(k_out=_H(5, 2, 64, dev=1)), dict(q_out=_H(5, 4, 64, dtype=F))]:
        with pytest.raises(ValueError):
            _norm(**bad)
    for bad in COMMON + [dict(dq_out=_H(5, 3, 64)), dict(dk=_H(5, 2, 64, dtype=F)), dict(dw_q=None), dict(dw_k=None),
                         dict(dw_q=[_T(63)]), dict(dw_q=[_T(64)] * 2), dict(dw_k=[_T(64, dtype=F)]), dict(rows=[0, 4]),
                         dict(ws=_T(1 << 20, dtype=torch.uint8, dev=1))]:
        with pytest.raises(ValueError):
            _norm_back(**bad)
    assert len(called) == 2


@pytest.mark.parametrize("name", ["embedding.cu", "qk_norm.cu", "token_logp.cu", "row_ops.cuh"])
def test_kernels_launched_behind_others_do_not_read_by_the_read_only_path(name):
    """As in test_sources_cpu.py: such a load's order against the wait for the kernel ahead is
    not defined."""
    with open(os.path.join(nb.CSRC, name)) as f:
        code = re.sub(r"//[^\n]*", "", f.read())
    assert "__ldg" not in code and not re.search(r"ld\.global(\.[a-z0-9:_]+)*\.nc", code) and "ld16_nc" not in code
