"""Tokens banned by a logit of -inf (a weight of -inf against a constant column): their
probability is 0, and everything else is as if they had the lowest finite logit."""
import pytest
import torch

from test_gpu_head_loss import check_loss, make
from paper_2608_01784_gb300 import api

pytestmark = pytest.mark.gpu
BANNED = [0, 7, 128, 300, 5999]


def banned(rows, k, vocab=6000, lowest=-float("inf")):
    h, w, t, grad = make(rows + k, rows, vocab, k, 0.8)
    w = w.clone()
    h[t >= 0, k - 1] = 1.0
    w[BANNED, k - 1] = lowest
    t = torch.where(torch.isin(t, torch.tensor(BANNED, device="cuda", dtype=torch.int32)), 1, t)
    return h, w, t, grad


@pytest.mark.parametrize("rows,k", [(1, 64), (32, 72), (40, 64), (64, 64), (65, 64), (500, 136)])
def test_loss(rows, k):
    h, w, t, _ = banned(rows, k)
    loss, lse = api.head_loss(h, w, t)
    check_loss(h, w, t, loss, lse)
    # a banned target: an infinite loss, the same lse
    live = t >= 0
    a, b = api.head_loss(h, w, torch.where(live, 7, t))
    assert bool((a[live] == float("inf")).all()) and torch.equal(b, lse)


@pytest.mark.parametrize("rows", [40, 64, 65])
def test_a_vocabulary_of_banned_tokens(rows):
    """All but one: it takes everything."""
    h, w, t, _ = banned(rows, 64)
    w[:, 63] = -float("inf")
    w[777, 63] = 0.0
    t = torch.where(t >= 0, 777, t)
    loss, lse = api.head_loss(h, w, t)
    live = t >= 0
    assert float(loss.abs().max()) == 0.0 and bool(lse[live].isfinite().all())
