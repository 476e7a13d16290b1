"""Log probabilities of rows of millions of logits against the formula in 64 bits, on the GPU."""
import math

import pytest
import torch

from test_token_logp_gpu import BF, DEV, F32, U, _forward, _Ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V", [1 << 27, (1 << 27) + 5])
def test_a_row_of_alike_logits(V):
    """One in 256 is 0, all the others are -1.4: nearly every addition to a sum of their powers is
    rounded to the same side."""
    x = float(torch.tensor(-1.4, dtype=F32))
    z = torch.full((1, V), x, device=DEV)
    z[torch.rand(1, V, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV) < 1 / 256] = 0.0
    first = (z[0] == 0).nonzero()[:, 0]
    n = first.numel()
    s = n + (V - n) * math.exp(x)
    L, far = math.log(s), -(V - n) * math.exp(x) * x / s
    # a logit's exponent is off by 3 roundings of |x|, 2^. by 4; at most 1100 additions (1024 and a few
    # single ones) make a sum that is put aside, at most 66 of which are added up; 60 to join threads
    s_err = U * (3 * abs(x) + 4 + 1100 + 66 + 60)
    for t in (int(first[-1]), 0):
        logp, stats, H, ids, top = _forward(z, torch.tensor([t], device=DEV), 3)
        lp = float(z[0, t]) - L
        assert abs(float(stats[0, 1]) - L) <= 1.01 * (s_err + 2 * U * L)
        assert abs(float(logp[0]) - lp) <= 1.01 * (s_err + 2 * U * (L + abs(x) + abs(lp)))
        assert abs(float(H[0]) - (L + far)) <= 1.01 * (s_err * (1 + 3 * (far + 1)) + 6 * U * (far * (abs(x) + 1) + L))
        assert torch.equal(ids[0], first[:3]) and bool((top[0] == top[0, 0]).all())


@pytest.mark.parametrize("dtype", [F32, BF])
def test_a_row_whose_beginning_is_ruled_out(dtype):
    """Most of what is put aside is nothing; the maximum comes late."""
    V = (1 << 25) + 3
    z = (torch.randn(2, V, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV) * 2).to(dtype)
    z[:, :3 * V // 4] = -math.inf
    z[1, :] = torch.sort(z[1]).values                # every thread's maximum rises all the way
    targets = torch.tensor([V - 5, V - 1], device=DEV)
    ref = _Ref(z, targets)
    ref.check(_forward(z, targets, 20), z)
    z[0, 7] = math.nan
    logp, stats, H, ids, top = _forward(z, targets, 2)
    assert bool(torch.isnan(logp[0])) and bool(torch.isnan(H[0])) and not bool(torch.isnan(logp[1]))
