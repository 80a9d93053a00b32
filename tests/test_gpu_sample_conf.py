"""The confidence of an unlikely token: as exact as fp32 takes it, however far its logit
lies below the largest."""
import pytest
import torch

from paper_2608_01784_gb300 import api
from tests.test_gpu_sample import BF16, F32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,vocab", [(150, 100), (150, 40000)])  # held, and walked
@pytest.mark.parametrize("filters", [{}, dict(temperature=0.9), dict(top_k=5)])
def test_confidence_of_unlikely_tokens(rows, vocab, dtype, filters):
    z = torch.full((rows, vocab), -float("inf"), device="cuda")
    z[:, 0] = torch.linspace(-19, -3, rows)   # token 0: u = 0 takes it
    z[:, vocab - 1] = 0.0
    z = z.to(dtype)
    kw = {n: torch.full((rows,), v, dtype=torch.int32 if n == "top_k" else F32, device="cuda")
          for n, v in filters.items()}
    tokens, conf = api.sample(z, torch.zeros(rows, device="cuda"), **kw)
    want = torch.softmax(z.double(), 1)[:, 0]
    assert bool((tokens == 0).all())
    # the exponential (2 ulp), the sum and the division (half an ulp each)
    assert bool(((conf.double() - want).abs() <= 3 * 2.0 ** -23 * want).all())
