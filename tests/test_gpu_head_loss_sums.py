"""The logits of the head's gradients are summed like those of its loss.

The tensor cores cut sums instead of rounding them, so sums of other lengths differ: of
positive products, 8192 of them in one sum, by 2e-4 for a logit of 40.  A row that is
sure of its target (every other logit lies 30 below) has lse = z and no gradient: the
other terms are below 700 exp(-30) = 7e-11 of its weight.  An exponential's exponent may
be off by 2^-24 of (|z| + |lse|) log2 e, and the exponential itself by 4 of its own
2^-24: TOL.  Gradients are products of that with one row of the operands, and rounded
once more."""
import pytest
import torch

from paper_2608_01784_gb300 import api

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
SURE = 40.0
TOL = (2 * (2 * SURE + 1) + 4) * U + 7e-11


@pytest.mark.parametrize("k", [600, 2048, 8192, 8200])
@pytest.mark.parametrize("rows,vocab", [(40, 6000), (200, 700)])
def test_gradients_of_sure_rows(rows, vocab, k):
    g = torch.Generator(device="cuda").manual_seed(rows + k)
    w = torch.randn(vocab, k, generator=g, device="cuda")
    w = (w / w.norm(dim=1, keepdim=True)).bfloat16()
    h = (SURE * w[:rows].float()).bfloat16()
    z = h.double() @ w.double().T
    at = torch.arange(rows, device="cuda")
    others = z.clone()
    others[at, at] = -1e9
    assert bool((others.amax(1) < z[at, at] - 30).all())  # (what the bound is made of)
    t = at.int()
    loss, lse = api.head_loss(h, w, t)
    dh = torch.empty(rows, k, device="cuda")
    dw = torch.empty(vocab, k, device="cuda")
    api.head_loss_backward(h, w, t, lse, torch.ones(rows, device="cuda"), d_hidden=dh, d_weight=dw)
    assert float((dh.abs() / w[:rows].float().abs().amax(1, keepdim=True)).max()) <= TOL
    # a token's gradient: its own row's term, and exp(-30) of the others
    size = h.float().abs().amax()
    assert float(dw.abs().max() / size) <= TOL
