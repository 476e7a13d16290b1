"""The gated projections on the GPU where values are extreme."""
import math

import pytest
import torch

from paper_2606_05613_gb300 import native as bk

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _phi(a):
    """Phi(a) (torch.special.ndtr is 0 from -8.3 down)."""
    return 0.5 * torch.special.erfc(-a * math.sqrt(0.5))


def _slope(name, a):
    """act'(a) in 64 bits, of any finite a."""
    if name == "silu":
        s = torch.sigmoid(a)
        return s + a * s * (1 - s)
    if name == "gelu":
        return _phi(a) + a * torch.exp(-a * a / 2) / math.sqrt(2 * math.pi)
    z = math.sqrt(2 / math.pi) * (a + 0.044715 * a ** 3)
    s = torch.sigmoid(2 * z)
    return s + 2 * a * s * (1 - s) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * a ** 2)


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("F", [64, 61])
def test_slopes_of_large_gates(act, F):
    """Gates of any finite bfloat16: the slope is 0 or 1 there, and da and db, which the call
    leaves in its workspace, are finite and right."""
    T, D = 8, 16
    size = torch.logspace(0, 38, T * F // 2 + 1, base=10.0, dtype=torch.float64, device=DEV)[:T * F // 2]
    a = torch.cat([size, -size, torch.zeros(T * F % 2, device=DEV, dtype=torch.float64)]).view(T, F).bfloat16()
    ld = (F + 7) // 8 * 8

    def rows(t):
        return torch.zeros(t.shape[0], ld, dtype=torch.bfloat16, device=DEV)[:, :F].copy_(t)

    one = torch.ones(T, F, device=DEV)
    x, w = torch.ones(T, D, dtype=torch.bfloat16, device=DEV), torch.ones(F, D, dtype=torch.bfloat16, device=DEV)
    ws = torch.zeros(bk.bkmoo_gate_backward_workspace_size(T, F), dtype=torch.uint8, device=DEV)
    bk.bkmoo_gate_backward(rows(0.5 * one), rows(a), rows(2.0 * one), x, w, w, act, [0, T], dx=torch.empty_like(x), ws=ws)
    da, db = (ws[i * ws.numel() // 2:][:T * ld * 2].view(torch.bfloat16).view(T, ld)[:, :F].double() for i in (0, 1))
    wide = a.double()
    f = wide * (_phi(wide) if act == "gelu" else torch.sigmoid(
        wide if act == "silu" else 2 * math.sqrt(2 / math.pi) * (wide + 0.044715 * wide ** 3)))
    # a bf16 rounding, the fast activation of terms up to 1.2, and what fp32 takes for 0
    assert bool(((da - _slope(act, wide)).abs() <= 2.0 ** -8 * 1.2 + 2.0 ** -17).all())
    assert bool(((db - 0.5 * f).abs() <= (2.0 ** -8 + 2.0 ** -17) * f.abs() + 1e-35).all())
