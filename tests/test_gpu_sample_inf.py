"""Greedy rows whose largest logit is +inf and whose finite ones are zeros or less:
the first +inf is taken, whatever the others are."""
import numpy as np
import pytest
import torch

from paper_2608_01784_gb300 import api
from tests.test_gpu_sample import BF16, F32, check, uniforms

pytestmark = pytest.mark.gpu
INF = float("inf")


def rows_of(n, vocab, dtype):
    g = torch.Generator().manual_seed(vocab)
    kinds = torch.zeros(5, vocab)
    kinds[0, vocab // 4] = INF
    kinds[1] = -0.0
    kinds[1, vocab - 1] = INF
    kinds[2] = -torch.rand(vocab, generator=g)
    kinds[2, ::7] = 0.0
    kinds[2, [vocab // 2, vocab // 2 + 1, vocab - 3]] = INF
    kinds[3, vocab // 3:] = float("nan")
    kinds[3, vocab - 2] = INF
    kinds[4] = -INF
    kinds[4, :vocab // 2] = 0.0
    kinds[4, vocab - 9] = INF
    return kinds.repeat(-(-n // 5), 1)[:n].to(dtype).cuda()


# a CTA a row, a cluster a row, and enough long rows to be walked in global memory
@pytest.mark.parametrize("rows,vocab", [(5, 2000), (500, 1999), (5, 50001), (90, 60001)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_the_first_infinity_is_taken(rows, vocab, dtype):
    z = rows_of(rows, vocab, dtype)
    u = uniforms(1, rows)
    check(z, u, T=np.zeros(rows, np.float32))
    tokens, conf = api.sample(z, torch.tensor(u, device="cuda"),
                              temperature=torch.zeros(rows, device="cuda"))
    inf = z == INF
    assert torch.equal(tokens.long(), inf.to(torch.uint8).argmax(1))
    assert torch.equal(conf, 1.0 / inf.sum(1).float())
    # greedy and sampled rows side by side
    T = np.where(np.arange(rows) % 2, 0.0, 0.7).astype(np.float32)
    check(z, u, T=T, k=np.full(rows, 3), p=np.full(rows, 0.9, np.float32))
