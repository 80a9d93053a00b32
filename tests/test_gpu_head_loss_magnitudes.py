"""Logits far from 0: exponents are taken of differences, which stay exact.

Rows of one large logit L and zeros (a column of h times one row of w), so that in fp32
lse = L and the loss of its target is 0, whatever L is, and the gradient there is
exp(z - lse) - 1 = 0; of two equal ones the loss is log 2.  Tolerances, with u = 2^-24: a
few roundings of the result itself, and 4 u for an exponential or logarithm near 1."""
import math

import pytest
import torch

from paper_2608_01784_gb300 import api

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
VOCAB, K = 6000, 64


def make(rows, size, top):
    """Row r has the logit L[r] in the columns `top`, 0 elsewhere."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    L = ((1 + torch.rand(rows, generator=g, device="cuda")) * size).bfloat16()
    h = torch.zeros(rows, K, device="cuda", dtype=torch.bfloat16)
    h[:, 3] = L
    w = torch.zeros(VOCAB, K, device="cuda", dtype=torch.bfloat16)
    w[top, 3] = 1.0
    return h, w, L.double()


@pytest.mark.parametrize("size", [30.0, 1e3, 1e5, 1e6, 1e7, 1e8, 1e12, 1e30])
@pytest.mark.parametrize("rows", [50, 300])
def test_one_large_logit(rows, size):
    h, w, L = make(rows, size, [4321])
    sure = torch.full((rows,), 4321, dtype=torch.int32, device="cuda")
    rest = VOCAB * math.exp(-size)  # of the zeros
    loss, lse = api.head_loss(h, w, sure)
    assert float(loss.abs().max()) <= 4 * U + rest
    assert bool(((lse.double() - L).abs() <= 4 * U * L + rest).all())
    other, same = api.head_loss(h, w, torch.zeros_like(sure))
    assert torch.equal(same, lse)
    assert bool(((other.double() - L).abs() <= 4 * U * L + rest).all())
    # and its gradients
    one = torch.ones(rows, device="cuda")
    dh, dw = api.head_loss_backward(h, w, sure, lse, one)
    assert float(dh.abs().max()) <= 4 * U + rest
    assert float(dw.abs().max()) <= (4 * U + rest) * float(L.sum())


@pytest.mark.parametrize("size", [1e5, 1e6, 1e7, 1e8, 1e12])
@pytest.mark.parametrize("rows", [50, 300])
def test_two_equal_large_logits(rows, size):
    """In slices of the vocabulary far from each other, and next to each other."""
    for top in ([11, 5999], [100, 101]):
        h, w, L = make(rows, size, top)
        loss, lse = api.head_loss(h, w, torch.full((rows,), top[1], dtype=torch.int32, device="cuda"))
        assert float((loss.double() - math.log(2)).abs().max()) <= 8 * U
        assert bool(((lse.double() - L - math.log(2)).abs() <= 4 * U * L).all())


@pytest.mark.parametrize("size", [1e5, 1e7, 1e8])
@pytest.mark.parametrize("rows", [50, 300])
def test_large_negative_logits(rows, size):
    """All logits but two are -L: those two carry the sum."""
    h, w, L = make(rows, -size, slice(None))
    w[[17, 3001], 3] = 0.0
    loss, lse = api.head_loss(h, w, torch.full((rows,), 17, dtype=torch.int32, device="cuda"))
    assert float((loss.double() - math.log(2)).abs().max()) <= 8 * U
    assert float((lse.double() - math.log(2)).abs().max()) <= 8 * U
