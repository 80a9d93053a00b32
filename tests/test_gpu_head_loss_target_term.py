"""The term of a row's target in the gradients is not rounded to bf16 with the rest of G.

It outweighs a row's other terms, and with few rows, or rows of one weight, nothing
averages its rounding out: at a weight of 1 + 2^-8, half way between two numbers of bf16,
the whole gradient was off by 2^-8.  Bounds as in test_gpu_head_loss, but half a step of
bf16 for the other terms alone (in the weights' gradient also for a token's rows behind
its fourth): the target's is off by the exponential and a few roundings of fp32, DELTA of
p and 4 u of itself, like any sum."""
import pytest
import torch

from test_gpu_head_loss import U, formula, make
from paper_2608_01784_gb300 import api

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def check(h, w, t, grad, dh, dw):
    i, z, lse = formula(h, w, t)
    n = i.numel()
    at, ti = torch.arange(n, device="cuda"), t[i].long()
    p, c, hd, wd = torch.exp(z - lse[:, None]), grad[i].double()[:, None], h[i].double(), w.double()
    off = c * p * (8 + 4 * (z.abs() + lse[:, None].abs())) * U
    p[at, ti] -= 1
    G = c * p
    size = G.abs()
    half = size * 2.0 ** -8
    fourth = torch.zeros(n, dtype=torch.bool, device="cuda")
    for j in range(n):
        fourth[j] = (ti[:j] == ti[j]).sum() < 4
    exact = half.clone()
    exact[at, ti] = 4 * U * size[at, ti]
    exact_w = half.clone()
    exact_w[at[fourth], ti[fourth]] = 4 * U * size[at[fourth], ti[fourth]]
    for got, ref, mag, terms, rounds in (
            (dh[i], G @ wd, lambda e: e @ wd.abs(), w.shape[0], exact),
            (dw, G.T @ hd, lambda e: e.T @ hd.abs(), n, exact_w)):
        bound = mag(rounds + size * 2 * terms * U + off) + torch.finfo(got.dtype).eps / 2 * ref.abs()
        assert float(((got.double() - ref).abs() - bound).max()) <= 0


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,vocab,k", [(1, 3000, 64), (1, 3000, 2047), (5, 900, 72), (33, 2500, 136),
                                          (64, 5000, 64), (65, 5000, 1001), (300, 700, 600),
                                          (300, 40, 64), (40, 30, 65), (700, 90, 264)])
def test_half_way_between_numbers(rows, vocab, k, dtype):
    h, w, t, grad = make(rows + vocab + k, rows, vocab, k, 0.9)
    grad = torch.where(t >= 0, 1 + 2.0 ** -8, float("nan"))
    _, lse = api.head_loss(h, w, t)
    dh = torch.full((rows, k), 7.0, device="cuda", dtype=dtype)
    dw = torch.full((vocab, k), 7.0, device="cuda", dtype=dtype)
    api.head_loss_backward(h, w, t, lse, grad, d_hidden=dh, d_weight=dw)
    check(h, w, t, grad, dh, dw)


@pytest.mark.parametrize("rows,vocab,k", [(8192, 9001, 40), (20000, 14000, 64), (3, 1050000, 16)])
def test_several_pieces(rows, vocab, k):
    h, w, t, _ = make(rows, rows, vocab, k, 0.3)
    grad = torch.where(t >= 0, 1 + 2.0 ** -8, float("nan"))
    _, lse = api.head_loss(h, w, t)
    dh = torch.empty(rows, k, device="cuda")
    dw = torch.empty(vocab, k, device="cuda")
    api.head_loss_backward(h, w, t, lse, grad, d_hidden=dh, d_weight=dw)
    check(h, w, t, grad, dh, dw)
    if rows > 3:
        return
    # relative errors over the whole: the other terms' rounding alone, where 2^-8 of all of it
    # would be 4e-3 (these rows know little: p < 0.01)
    i, z, ref = formula(h, w, t)
    p = torch.exp(z - ref[:, None])
    assert float(p.max()) < 0.01
    p[torch.arange(i.numel()), t[i].long()] -= 1
    G = (1 + 2.0 ** -8) * p
    for got, r in ((dh[i], G @ w.double()), (dw, G.T @ h[i].double())):
        assert float((got.double() - r).norm() / r.norm()) <= 1e-3


def test_an_infinite_weight_of_the_target():
    """A banned target: its row's gradient is infinite there, and no NaN more than the
    formula has; a token that nobody has stays at 0."""
    h, w, t, grad = make(3, 40, 900, 64)
    w = w.clone()
    h[:, 63] = 1.0
    w[5, 63] = -float("inf")
    t.fill_(7)
    t[3] = 5
    loss, lse = api.head_loss(h, w, t)
    assert float(loss[3]) == float("inf")
    dh, dw = api.head_loss_backward(h, w, t, lse, torch.ones(40, device="cuda"))
    assert float(dh[3, 63]) == float("inf") and bool(dh[3, :63].isfinite().all())
    assert bool(dw.isfinite().all())
