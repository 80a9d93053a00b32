"""Sampling at the ends of its settings: rows that masks leave one logit of, and the
largest temperatures."""
import numpy as np
import pytest
import torch

from paper_2608_01784_gb300 import _binding as B
from paper_2608_01784_gb300 import api
from tests.test_gpu_sample import BF16, F32

pytestmark = pytest.mark.gpu
LARGEST = float(np.finfo(np.float32).max)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,vocab", [(3, 1000), (3, 262144), (90, 262144)])
@pytest.mark.parametrize("other", [-float("inf"), float("nan"), -1e9])
def test_the_only_token_has_confidence_one(rows, vocab, dtype, other):
    """Nothing of the tokens that a mask left out is in the softmax's sum."""
    z = torch.full((rows, vocab), other, dtype=dtype, device="cuda")
    at = torch.arange(rows, device="cuda") * 7 % vocab
    z[torch.arange(rows), at] = 0.5
    tokens, conf = api.sample(z, torch.full((rows,), 0.3, device="cuda"))
    assert torch.equal(tokens.long(), at)
    assert bool((conf == 1.0).all()), float(conf.min())


@pytest.mark.parametrize("T", [3.4e38, LARGEST])
def test_every_finite_temperature(T):
    """The logits vanish beside it: evenly spaced uniforms walk the vocabulary."""
    n = 64
    z = torch.randn(1, n, generator=torch.Generator().manual_seed(1)).expand(n, n).contiguous().cuda()
    u = (torch.arange(n, device="cuda") + 0.5) / n
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    tokens, conf = api.sample(z, u, temperature=torch.full((n,), T, device="cuda"), status=status)
    assert B.reflex_read_status(status) == B.REFLEX_OK
    assert torch.equal(tokens.cpu(), torch.arange(n, dtype=torch.int32))
    assert bool((conf > 0).all())
