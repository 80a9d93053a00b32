"""Up to 64 rows a row's loss has the same bits wherever it stands and whatever stands
around it: the rows of W are added up in one order.  A constant column keeps lse near 0,
where its last bits show."""
import pytest
import torch

from paper_2608_01784_gb300 import api

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("vocab,k", [(6000, 96), (20001, 64), (131072, 128)])
def test_the_same_bits(vocab, k):
    g = torch.Generator(device="cuda").manual_seed(vocab)
    h = torch.randn(64, k, generator=g, device="cuda").bfloat16()
    w = (torch.randn(vocab, k, generator=g, device="cuda") * k ** -0.5).bfloat16()
    h[:, 0] = 1.0
    w[:, 0] = -torch.log(torch.tensor(float(vocab))) - 0.5
    t = torch.randint(0, vocab, (64,), generator=g, device="cuda", dtype=torch.int32)
    loss, lse = api.head_loss(h, w, t)
    assert float(lse.abs().max()) < 1.0
    for lo, hi in ((0, 1), (0, 31), (0, 32), (0, 33), (31, 64), (32, 64), (40, 41), (13, 45), (7, 60)):
        a, b = api.head_loss(h[lo:hi], w, t[lo:hi].contiguous())
        assert torch.equal(a, loss[lo:hi]) and torch.equal(b, lse[lo:hi]), (lo, hi)
    # other places: every second row left out, and another order
    half = t.clone()
    half[::2] = -1
    a, b = api.head_loss(h, w, half)
    assert torch.equal(a[1::2], loss[1::2]) and torch.equal(b[1::2], lse[1::2])
    p = torch.randperm(64, generator=g, device="cuda")
    a, b = api.head_loss(h[p], w, t[p])
    assert torch.equal(a, loss[p]) and torch.equal(b, lse[p])
