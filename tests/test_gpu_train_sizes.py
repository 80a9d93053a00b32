"""Sizes that do not fit the library's 32 bits are refused, not cut to what fits.  (Cut,
each of these would be an ordinary small call.)"""
import pytest
import torch

from paper_2608_01784_gb300 import _binding as B
from paper_2608_01784_gb300 import api

pytestmark = pytest.mark.gpu
CUT = 2 ** 32  # a multiple of it is lost
BF16 = torch.bfloat16


@pytest.fixture(autouse=True)
def nothing_enqueued(monkeypatch):
    def enqueued(*args, **kw):
        raise AssertionError("the call went on")
    for name in B.EXPORTED[B.EXPORTED.index("reflex_block_norm"):]:
        if not name.endswith("_workspace_size"):
            monkeypatch.setattr(B, name, enqueued)


@pytest.fixture(scope="module")
def memory():
    return torch.empty(CUT + 64, dtype=BF16, device="cuda")


def test_wide_rows(memory):
    x = memory[:CUT + 8].view(1, CUT + 8)
    plan = api.ExpertPlan(1, 4, 1, 1, x.device)
    one = torch.ones(1, 1, device="cuda")
    calls = [lambda: api.block_norm(x, out=x), lambda: api.block_norm(x, x, out=x),
             lambda: api.block_norm_backward(x, None, x, None, d_h=x),
             lambda: api.expert_rows(x, plan, rows=x), lambda: api.expert_rows_backward(x, plan, out=x),
             lambda: api.expert_combine(x, one, plan, out=x),
             lambda: api.expert_combine_backward(x, x, one, plan, d_rows=x)]
    for i, c in enumerate(calls):
        with pytest.raises(ValueError):
            c()
            pytest.fail(f"call {i} went on")


def test_heads(memory):
    tall = memory[:CUT + 8].view(CUT + 8, 1)  # as hidden rows, and as columns of the weights
    row = memory[:CUT + 8].view(1, CUT + 8)
    few = torch.zeros(8, dtype=torch.int32, device="cuda")
    many = few[:1].expand(CUT + 8)
    lse = torch.zeros(8, device="cuda")
    weight = torch.zeros(16, 8, dtype=BF16, device="cuda")[:, :1]
    for call in (lambda: api.head_loss(tall, weight, few), lambda: api.head_loss(tall, weight, many),
                 lambda: api.head_loss(row, row, few[:1]),
                 lambda: api.head_loss_backward(row, row, few[:1], lse[:1], lse[:1])):
        with pytest.raises(ValueError):
            call()
            pytest.fail("a call went on")


@pytest.mark.parametrize("E", [CUT + 8, 2 ** 31, 1025, 0, -8])
def test_plans(E):
    ids = torch.zeros(4, 2, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        api.expert_plan(ids, E=E)
