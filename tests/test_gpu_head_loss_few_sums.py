"""Up to 64 rows, sums of 256 products are added to the nearest.

A token's logit of one product of 8 and 511 of 15 2^-28: sixteen of them, which the tensor
cores take at a time, are 15/16 of a step of 8 (2^-20), and may be cut off every time, 16
times in a sum of 256.  The other 256 come in a sum of their own, where a step is far
smaller, and are added with half a step.  Against 2981 tokens of logit 0 the token weighs
as much as all of them; the target is one of the others."""
import math

import pytest
import torch

from paper_2608_01784_gb300 import api

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
VOCAB, K = 2982, 512


@pytest.mark.parametrize("rows", [1, 32, 33, 64])
def test_a_large_logit_that_is_not_the_target(rows):
    h = torch.full((rows, K), 2.0 ** -14, device="cuda", dtype=torch.bfloat16)
    h[:, 0] = 1.0
    w = torch.zeros(VOCAB, K, device="cuda", dtype=torch.bfloat16)
    w[77] = 15 * 2.0 ** -14
    w[77, 0] = 8.0
    t = torch.full((rows,), 500, dtype=torch.int32, device="cuda")
    z = 8.0 + (K - 1) * 15 * 2.0 ** -28
    lse = math.log(math.exp(z) + VOCAB - 1)
    loss, got = api.head_loss(h, w, t)
    p = math.exp(z - lse)
    tol = p * (16 + 0.5) * 2.0 ** -20 + 8 * U + 4 * U * lse  # (one exponential and its sum)
    assert float((got.double() - lse).abs().max()) <= tol
    assert float((loss.double() - lse).abs().max()) <= tol
