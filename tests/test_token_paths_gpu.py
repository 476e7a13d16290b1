"""Sizes that take the operators on tokens through steps that test_qk_norm_gpu.py and
test_embedding_gpu.py leave out, by the checks of those, on the GPU."""
import pytest
import torch

import test_embedding_gpu as embedding
import test_qk_norm_gpu as norms

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32

# narrow heads, more than a warp takes at once: 32 of 16 or 16 of 32 elements; steps of queries alone, of
# both, of keys alone
NARROW = [
    # T, hq, hk, hd, rot, interleaved, K, w dtype, ld beyond the heads, far
    (40, 70, 35, 16, 16, False, 3, BF, 0, True),
    (40, 70, 35, 16, 16, True, 3, BF, 8, False),
    (70, 64, 32, 16, 16, False, 4, F32, 0, False),
    (40, 37, 5, 32, 32, False, 3, BF, 0, True),
    (40, 37, 40, 32, 16, True, 3, F32, 16, False),
    (33, 16, 16, 32, 0, False, 2, BF, 0, False),
]


@pytest.mark.parametrize("case", NARROW)
def test_narrow_heads_normed_and_rotated(case):
    norms.test_normed_and_rotated(case)


@pytest.mark.parametrize("accumulate,out", [(False, BF), (True, F32)])
@pytest.mark.parametrize("case", NARROW)
def test_gradients_of_narrow_heads(case, accumulate, out):
    norms.test_gradients_by_language(case, accumulate, out)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("T,V,K,distinct", [(300000, 500, 3, 2), (300000, 1 << 19, 2, 1 << 19), (262145, 70, 1, 70),
                                            (262144, 70, 4, 70)])
def test_gradients_of_rows_in_order_by_four_kernels(T, V, K, distinct, accumulate):
    """Runs of 256 rows are merged 32 at a time: from 262145 rows on three times."""
    embedding.test_gradients_by_token_and_language(T, V, 8, K, distinct, 8, 0, BF, F32, accumulate)
