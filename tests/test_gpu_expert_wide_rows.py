"""Rows of 2 GB and more: their bytes pass 31 bits."""
import pytest
import torch

from paper_2608_01784_gb300 import api

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d", [(torch.float32, (1 << 29) + 4), (torch.float32, (1 << 29) + 1),
                                     (torch.bfloat16, 1 << 30), (torch.bfloat16, (1 << 30) - 2),
                                     (torch.float32, 1 << 30)])
def test_one_token(dtype, d):
    x = torch.arange(d, device="cuda", dtype=torch.int32).remainder_(251).to(dtype).view(1, d)
    plan = api.expert_plan(torch.tensor([[1]], dtype=torch.int32, device="cuda"), E=2)
    rows = torch.full((1, d), -1.0, device="cuda", dtype=dtype)
    api.expert_rows(x, plan, rows=rows)
    assert torch.equal(rows, x)
    alpha = torch.full((1, 1), 2.0, device="cuda")
    out = torch.full((1, d), -1.0, device="cuda", dtype=dtype)
    api.expert_combine(rows, alpha, plan, out=out)
    assert torch.equal(out, x.mul_(2))
    d_rows, d_alpha = api.expert_combine_backward(out, rows, alpha, plan, d_rows=torch.zeros_like(x))
    assert torch.equal(d_rows, x.mul_(2)) and bool(d_alpha.isfinite().all())
