"""The target's logit, which a loss is the difference to, is summed to the nearest.

One product of 8 and K - 1 of 2^-22: tensor cores drop the small ones next to the large
one (2^-25 of it), up to 511 of them in a sum of 512.  In the kernel that adds up the target's
logit only the 7 (or, with the rows of a lane, the first of each eight) products next to the
large one can be lost to rounding, then sums of eights are exact up to a rounding of 2^-24 of
8 each: LOST.  All other logits are 0; exp(8) = 2981 of them weigh as much as the target."""
import math

import pytest
import torch

from paper_2608_01784_gb300 import api

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
VOCAB = 2982


@pytest.mark.parametrize("k", [512, 1000, 2047, 2048, 4096, 5000])
@pytest.mark.parametrize("rows", [1, 40, 64, 65, 300, 700])
def test_loss_and_gradients(rows, k):
    h = torch.full((rows, k), 2.0 ** -11, device="cuda", dtype=torch.bfloat16)
    h[:, 0] = 1.0
    ld = -(-k // 8) * 8
    w = torch.zeros(VOCAB, ld, device="cuda", dtype=torch.bfloat16)[:, :k]
    w[77] = 2.0 ** -11
    w[77, 0] = 8.0
    t = torch.full((rows,), 77, dtype=torch.int32, device="cuda")
    z = 8.0 + (k - 1) * 2.0 ** -22
    lost = (-(-k // 256) + 5) * 8 * U + 7 * 2.0 ** -22
    lse = math.log(math.exp(z) + VOCAB - 1)
    p = math.exp(z - lse)
    loss, got = api.head_loss(h, w, t)
    tol = lost + (64 + VOCAB / 2048) * U + 4 * U * lse  # (that of test_gpu_head_loss)
    assert float((got.double() - lse).abs().max()) <= tol
    assert float((loss.double() - (lse - z)).abs().max()) <= tol
    dh = torch.empty(rows, k, device="cuda")
    api.head_loss_backward(h, w, t, got, torch.ones(rows, device="cuda"), d_hidden=dh, need_weight=False)
    want = (p - 1) * 8.0
    assert float((dh[:, 0].double() - want).abs().max()) <= 8.0 * (p * 2 * tol + 8 * U)


def test_the_same_bits_in_calls_of_any_size():
    """The sum's order depends neither on how many rows there are nor on how they lie."""
    g = torch.Generator(device="cuda").manual_seed(3)
    rows, vocab, k = 1500, 900, 520
    h = torch.randn(rows, k, generator=g, device="cuda").bfloat16()
    w = (torch.randn(vocab, k, generator=g, device="cuda") * 0.1).bfloat16()
    t = torch.randint(0, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
    grad = torch.rand(rows, generator=g, device="cuda")
    odd = torch.zeros(rows * (k + 1) + 1, device="cuda", dtype=torch.bfloat16)[1:].view(rows, k + 1)[:, :k]
    odd.copy_(h)
    loss, lse = api.head_loss(h, w, t)
    dh, _ = api.head_loss_backward(h, w, t, lse, grad, need_weight=False)
    a, b = api.head_loss(odd, w, t)
    assert torch.equal(a, loss) and torch.equal(b, lse)
    for lo, hi in ((0, 100), (200, 504), (200, 505), (700, 1500)):
        part = slice(lo, hi)
        a, b = api.head_loss(h[part], w, t[part].contiguous())
        assert torch.equal(a, loss[part]) and torch.equal(b, lse[part])
        a, _ = api.head_loss_backward(h[part], w, t[part].contiguous(), b, grad[part].contiguous(),
                                      need_weight=False)
        # (parts of the vocabulary depend on the number of rows: the sums behind the terms differ)
        assert float((a.double() - dh[part].double()).norm() / dh[part].double().norm()) <= 2.0 ** -8
