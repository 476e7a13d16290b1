"""CPU: the operators' entry points refuse bad arguments before they touch a
GPU, and the host-only parts.  Addresses are made up and never read."""
import ctypes
import math

import pytest
import torch

from paper_2606_05613_gb300 import build as nb
from paper_2606_05613_gb300 import native as bk

OK, INVALID, WS = bk.BKMOO_OK, bk.BKMOO_ERR_INVALID, bk.BKMOO_ERR_WORKSPACE
P = 1 << 40                       # an aligned address


@pytest.fixture(scope="module", autouse=True)
def _built():
    nb.build()
    bk.load()


def _forward(**k):
    a = dict(x=P, ldx=64, wg=P, wu=P, ldw=64, T=5, D=64, F=128, act=0, h=P, ldh=128, a=P, b=P, ld_ab=128)
    a.update(k)
    return bk.load().bkmoo_gate_forward(a["x"], a["ldx"], a["wg"], a["wu"], a["ldw"], a["T"], a["D"], a["F"], a["act"],
                                        a["h"], a["ldh"], a["a"], a["b"], a["ld_ab"], None)


@pytest.mark.parametrize("bad", [dict(act=3), dict(act=-1), dict(T=-1), dict(D=0), dict(F=0), dict(x=None), dict(wg=None),
                                 dict(wu=None), dict(h=None, a=None, b=None), dict(a=None), dict(b=None), dict(x=P + 8),
                                 dict(wg=P + 2), dict(h=P + 4), dict(a=P + 8), dict(ldx=63), dict(ldx=68), dict(ldw=56),
                                 dict(ldh=120), dict(ldh=132), dict(ld_ab=64), dict(T=1 << 31), dict(F=1 << 33),
                                 dict(D=1 << 33, ldx=1 << 33, ldw=1 << 33), dict(T=1 << 30, D=1 << 20, ldx=1 << 20, ldw=1 << 20)])
def test_forward_refuses(bad):
    assert _forward(**bad) == INVALID


def test_forward_without_rows_does_nothing():
    assert _forward(T=0, x=None, h=None, a=None, b=None) == OK


def _rows(*r):
    return (ctypes.c_int64 * len(r))(*r)


def _ptrs(*p):
    return (ctypes.c_void_p * len(p))(*p)


def _backward(**k):
    a = dict(dh=P, ld_dh=128, a=P, b=P, ld_ab=128, x=P, ldx=64, wg=P, wu=P, ldw=64, T=5, D=64, F=128, act=0, K=2,
             rows=_rows(0, 2, 5), dx=P, ld_dx=64, dg=_ptrs(P, P), du=_ptrs(P, P), dt=1, acc=0, ws=P, nb=1 << 30)
    a.update(k)
    return bk.load().bkmoo_gate_backward(a["dh"], a["ld_dh"], a["a"], a["b"], a["ld_ab"], a["x"], a["ldx"], a["wg"], a["wu"],
                                         a["ldw"], a["T"], a["D"], a["F"], a["act"], a["K"], a["rows"], a["dx"], a["ld_dx"],
                                         a["dg"], a["du"], a["dt"], a["acc"], a["ws"], a["nb"], None)


@pytest.mark.parametrize("bad", [dict(act=7), dict(T=-1), dict(dt=2), dict(dt=-1), dict(K=0), dict(K=17), dict(rows=None),
                                 dict(rows=_rows(1, 2, 5)), dict(rows=_rows(0, 2, 4)), dict(rows=_rows(0, 6, 5)),
                                 dict(dx=None, dg=None, du=None), dict(dg=None), dict(du=None), dict(dg=_ptrs(P, None)),
                                 dict(du=_ptrs(P, P + 1)), dict(dt=0, dg=_ptrs(P, P + 2)), dict(dh=None), dict(a=None),
                                 dict(b=None), dict(x=None), dict(dh=P + 8), dict(ld_dh=127), dict(ld_dx=60), dict(dx=P + 2),
                                 dict(ws=None), dict(ws=P + 128), dict(D=1 << 20, F=1 << 20, ldx=1 << 20, ldw=1 << 20)])
def test_backward_refuses(bad):
    assert _backward(**bad) == INVALID


def test_backward_needs_its_workspace():
    n = bk.bkmoo_gate_backward_workspace_size(5, 128)
    assert _backward(nb=n - 1) == WS
    assert n == 2 * 1280 and bk.bkmoo_gate_backward_workspace_size(37, 2731) == 2 * math.ceil(37 * 2736 * 2 / 256) * 256
    assert bk.bkmoo_gate_backward_workspace_size(0, 8) == 0
    for T, F in ((-1, 8), (4, 0)):
        with pytest.raises(bk.BkmooError):
            bk.bkmoo_gate_backward_workspace_size(T, F)


def _wgrad(**k):
    a = dict(dy=P, ld_dy=128, x=P, ldx=64, T=5, M=128, N=64, K=2, rows=_rows(0, 2, 5), dw=_ptrs(P, P), dt=0, acc=0)
    a.update(k)
    return bk.load().bkmoo_language_wgrad(a["dy"], a["ld_dy"], a["x"], a["ldx"], a["T"], a["M"], a["N"], a["K"], a["rows"],
                                          a["dw"], a["dt"], a["acc"], None)


@pytest.mark.parametrize("bad", [dict(T=-1), dict(M=0), dict(N=0), dict(K=0), dict(K=17), dict(rows=None), dict(dw=None),
                                 dict(rows=_rows(0, 3, 2)), dict(dw=_ptrs(P, P + 2)), dict(dt=2), dict(dy=None), dict(x=None),
                                 dict(dy=P + 8), dict(ldx=60), dict(ld_dy=120), dict(M=1 << 20, N=1 << 20)])
def test_wgrad_refuses(bad):
    assert _wgrad(**bad) == INVALID


def _adamw(p=None, **k):
    q = bk.bkmoo_adamw_default_params()
    for name, v in (p or {}).items():
        setattr(q, name, v)
    a = dict(ts=_ptrs(P, P), sizes=_rows(10, 20), wd=None, n=2, pd=0, g=P, gd=0, master=None, m=P, v=P, ms=P, vs=P, sd=0,
             q=ctypes.byref(q), norm=P)
    a.update(k)
    return bk.load().bkmoo_adamw(a["ts"], a["sizes"], a["wd"], a["n"], a["pd"], a["g"], a["gd"], a["master"], a["m"], a["v"],
                                 a["ms"], a["vs"], a["sd"], a["q"], a["norm"], None)


def _decay(*d):
    return (ctypes.c_float * len(d))(*d)


@pytest.mark.parametrize("bad", [dict(n=-1), dict(ts=None), dict(sizes=None), dict(pd=2), dict(gd=2), dict(sd=1), dict(sd=3),
                                 dict(q=None), dict(master=P), dict(sizes=_rows(10, -1)), dict(ts=_ptrs(P, None)),
                                 dict(ts=_ptrs(P, P + 2)), dict(wd=_decay(0.1, -0.1)), dict(wd=_decay(0.1, math.inf)),
                                 dict(g=None), dict(g=P + 8), dict(m=P + 4), dict(v=None), dict(pd=1, master=P + 8),
                                 dict(sd=2, ms=None), dict(sd=2, vs=P + 2), dict(sizes=_rows(1 << 47, 1 << 48)),
                                 dict(p=dict(beta1=1.0)), dict(p=dict(beta2=-0.1)), dict(p=dict(eps=-1.0)),
                                 dict(p=dict(lr=math.nan)), dict(p=dict(max_norm=-1.0)), dict(p=dict(step=0)),
                                 dict(p=dict(max_norm=1.0), norm=None), dict(p=dict(beta1=math.nan)), dict(norm=P + 2)])
def test_adamw_refuses(bad):
    assert _adamw(**bad) == INVALID


def test_adamw_without_elements_does_nothing():
    assert _adamw(n=0, ts=None, sizes=None) == OK
    assert _adamw(sizes=_rows(0, 0), ts=_ptrs(None, None), g=None, m=None, v=None) == OK


def test_adamw_defaults():
    p = bk.bkmoo_adamw_default_params()
    assert (p.lr, p.beta1, p.beta2, p.eps, p.max_norm, p.step, p.seed) == (1e-3, 0.9, 0.999, 1e-8, 0.0, 1, 0)


@pytest.mark.parametrize("bad", [dict(dt=2), dict(n=-1), dict(out=None), dict(out=P + 2), dict(ws=None), dict(ws=P + 64),
                                 dict(g=None), dict(g=P + 8)])
def test_norm_refuses(bad):
    a = dict(g=P, dt=0, n=5, out=P, ws=P, nb=bk.BKMOO_NORM_WS_BYTES)
    a.update(bad)
    call = bk.load().bkmoo_grad_norm
    assert call(a["g"], a["dt"], a["n"], a["out"], a["ws"], a["nb"], None) == INVALID
    assert call(P, 0, 5, P, P, bk.BKMOO_NORM_WS_BYTES - 1, None) == WS


def test_status_needs_a_place():
    assert bk.load().bkmoo_op_status(None, None) == INVALID


def test_binding_refuses_what_is_not_on_a_gpu():
    x, w = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(8, 64, dtype=torch.bfloat16)
    h = torch.zeros(4, 8, dtype=torch.bfloat16)
    for call in (lambda: bk.bkmoo_gate_forward(x, w, w, "silu", h),
                 lambda: bk.bkmoo_gate_backward(h, h, h, x, w, w, "silu", [0, 4], x),
                 lambda: bk.bkmoo_language_wgrad(x, x, [0, 4], [torch.zeros(64, 64)]),
                 lambda: bk.bkmoo_grad_norm(torch.zeros(8), torch.zeros(1)),
                 lambda: bk.bkmoo_adamw([torch.zeros(8)], torch.zeros(8), torch.zeros(8), torch.zeros(8)),
                 lambda: bk.TensorList([]),
                 lambda: bk.TensorList([torch.zeros(8)])):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("rows", [[0], [1, 4], [0, 3], [0, 5, 4], list(range(18)) + [4], [0] * 17 + [4, 4]])
def test_binding_refuses_language_bounds(rows):
    with pytest.raises(ValueError):
        bk._language_rows(rows, 4)
    assert bk._language_rows([0, 0, 4], 4)[0] == 2
