"""Every width of tile and way of writing of the gate and weight-gradient kernels on
the GPU, pairs of CTAs among them, against the formulas in 64 bits at the tolerances of
test_gate_gpu.py, with edges inside the tiles and an empty language (tile_shapes.py)."""
import math

import pytest
import torch

from paper_2606_05613_gb300 import native as bk
from test_gate_gpu import (HALF, _backward_ref, _check, _forward_ref, _framed, _grads, _mat, _room, _wgrad_ref)
from tile_shapes import BACKWARD, FORWARD, WGRAD, rows

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
WAYS = [(torch.bfloat16, False), (torch.bfloat16, True), (torch.float32, False), (torch.float32, True)]


def _around(flat, at, n):
    return all(bool((f[:at] == 5).all()) and bool((f[at + n:] == 5).all()) for f in flat)


@pytest.mark.parametrize("T,D,F,shape", FORWARD)
def test_forward(T, D, F, shape):
    gen = torch.Generator(device=DEV).manual_seed(T + D + F)
    x, wg, wu = _mat(gen, T, D, pad=3), _mat(gen, F, D, 1.5 / math.sqrt(D)), _mat(gen, F, D, 1 / math.sqrt(D))
    for act in ("silu", "gelu", "gelu_tanh"):
        refs = _forward_ref(x, wg, wu, act)
        (wh, h), (wa, a), (wb, b) = _room(T, F, pad=8), _room(T, F, lead=8), _room(T, F, lead=8)
        bk.bkmoo_gate_forward(x, wg, wu, act, h, a, b)
        for out, ref, name in zip((h, a, b), refs, "hab"):
            _check(out, ref[0], ref[1], (name, act))
        assert _framed(wh, h, 0) and _framed(wa, a, 8) and _framed(wb, b, 8)
        alone = _room(T, F)[1]
        bk.bkmoo_gate_forward(x, wg, wu, act, alone)
        assert torch.equal(alone, h)
    assert bk.bkmoo_op_status(DEV) == 0


@pytest.mark.parametrize("T,D,F,K", [c[:4] for c in BACKWARD])
def test_backward(T, D, F, K):
    gen = torch.Generator(device=DEV).manual_seed(T + D + F)
    x, wg, wu = _mat(gen, T, D), _mat(gen, F, D, 1 / math.sqrt(D)), _mat(gen, F, D, 1 / math.sqrt(D))
    a, b, dh = _mat(gen, T, F, 1.5, lead=8), _mat(gen, T, F, lead=8), _mat(gen, T, F, 0.1, pad=9)
    bounds = rows(T, K)
    (dx_ref, dx_err), g_ref, u_ref = _backward_ref(dh, a, b, x, wg, wu, "silu", bounds)
    for dtype, odd in WAYS:
        half = HALF if dtype == torch.bfloat16 else 2.0 ** -23
        for fill in (0.0, 0.75):                     # written, and added to that
            wdx, dx = _room(T, D, pad=8)
            (fg, dg, at), (fu, du, _) = _grads(K, F, D, dtype, odd, fill=fill), _grads(K, F, D, dtype, odd, fill=fill)
            bk.bkmoo_gate_backward(dh, a, b, x, wg, wu, "silu", bounds, dx, dg, du, accumulate=fill != 0.0)
            _check(dx, dx_ref, HALF * dx_ref.abs() + 1.02 * dx_err, ("dx", dtype, odd, fill))
            assert _framed(wdx, dx, 0) and _around(fg + fu, at, F * D)
            for k in range(K):
                for out, (ref, err) in ((dg[k], g_ref[k]), (du[k], u_ref[k])):
                    total = ref + fill
                    add = 2.0 ** -23 * total.abs() if fill else 0.0
                    _check(out, total, half * total.abs() + 1.02 * err + add, ("dw", k, dtype, odd, fill))
                    if bounds[k] == bounds[k + 1]:
                        assert bool((out == fill).all())
    assert bk.bkmoo_op_status(DEV) == 0


@pytest.mark.parametrize("T,M,N,K", [c[:4] for c in WGRAD])
def test_language_wgrad(T, M, N, K):
    gen = torch.Generator(device=DEV).manual_seed(T + M + N)
    dy, x = _mat(gen, T, M, 0.1, pad=5), _mat(gen, T, N)
    bounds = rows(T, K)
    ref, err = _wgrad_ref(dy, x, bounds)
    for dtype, odd in WAYS:
        half = HALF if dtype == torch.bfloat16 else 2.0 ** -23
        for fill in (0.0, 0.75):
            flat, dw, at = _grads(K, M, N, dtype, odd, fill=fill)
            bk.bkmoo_language_wgrad(dy, x, bounds, dw, accumulate=fill != 0.0)
            assert _around(flat, at, M * N)
            for k in range(K):
                total = ref[k] + fill
                add = 2.0 ** -23 * total.abs() if fill else 0.0
                _check(dw[k], total, half * total.abs() + 1.02 * err[k] + add, ("dw", k, dtype, odd, fill))
                if bounds[k] == bounds[k + 1]:
                    assert bool((dw[k] == fill).all())
    assert bk.bkmoo_op_status(DEV) == 0


@pytest.mark.parametrize("T,D,F,K", [c[:4] for c in BACKWARD if c[4] == "2x256"])
def test_pairs_give_the_same_bits_again(T, D, F, K):
    """Bounds and gradients that change from call to call, with nothing between the calls."""
    gen = torch.Generator(device=DEV).manual_seed(T)
    x, wg, wu = _mat(gen, T, D), _mat(gen, F, D, 0.05), _mat(gen, F, D, 0.05)
    a, b, dh = _mat(gen, T, F), _mat(gen, T, F), _mat(gen, T, F, 0.1)
    many = [rows(T, K), [0] * K + [T], [T * k // K for k in range(K + 1)]]
    seen = []
    for _ in range(2):
        dx = _room(T, D)[1]
        (_, dg, _), (_, du, _) = (_grads(K, F, D, torch.bfloat16, False, fill=0.75) for _ in range(2))
        h = _room(T, F)[1]
        for i in range(12):
            bk.bkmoo_gate_forward(x, wg, wu, "silu", h, a, b)
            bk.bkmoo_gate_backward(dh, a, b, x, wg, wu, "silu", many[i % 3], dx, dg, du, accumulate=i % 4 != 0)
        seen.append([t.clone() for t in [h, dx] + dg + du])
    assert all(torch.equal(u, v) for u, v in zip(*seen))
    assert bk.bkmoo_op_status(DEV) == 0
