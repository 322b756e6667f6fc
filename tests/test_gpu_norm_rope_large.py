"""The gradient of bc_norm_rope_split over millions of rows."""
import numpy as np
import pytest
import torch

from paper_2510_13797_b200 import binding as B
from tests.harness import f64

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("D", [64, 128])
def test_weight_gradients_over_millions_of_rows(D):
    """Equal terms, each a little more than a number that fp32 sums of a thousand of them can hold: a sum of 1700 in a row (a lane's terms
    here) would lose 388 times 2^-24.  Allowed: 128 additions per lane, 14 of these sums, 3 between lanes, 8 warps, 42 in the last
    kernel, and 8 roundings of the term itself: 203 times 2^-24."""
    n = 2368 * 1700
    qkv = torch.ones((n, 3 * D), dtype=torch.bfloat16, device=DEV)
    g = torch.full((n, 1, D), 1.0078125, dtype=torch.bfloat16, device=DEV)
    # the term x r g is to be 1 + 0.49 * 2^-13
    eps = float(np.float32((1.0078125 / (1 + 0.49 * 2.0 ** -13)) ** 2 - 1))
    pos = torch.zeros(n, dtype=torch.int32, device=DEV)
    dqkv, dwq, dwk = B.bc_norm_rope_split_backward(qkv, pos, 1e4, None, None, eps, g, g, g)
    want = n * 1.0078125 / np.sqrt(1 + eps)
    for dw in (dwq, dwk):
        assert np.abs(f64(dw) / want - 1).max() <= 203 * 2.0 ** -24
    dx = 1.0078125 / np.sqrt(1 + eps) * (1 - 1 / (1 + eps))
    assert (dqkv[:, :2 * D].amin().item(), dqkv[:, :2 * D].amax().item()) == (pytest.approx(dx, rel=2.0 ** -8 + 1e-4),) * 2
