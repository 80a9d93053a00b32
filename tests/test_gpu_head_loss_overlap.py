"""d_weight beside and over the weights, through the Python call."""
import pytest
import torch

from test_gpu_head_loss import check_grad, make
from paper_2608_01784_gb300 import _binding as B
from paper_2608_01784_gb300 import api

pytestmark = pytest.mark.gpu
ROWS, VOCAB, K = 70, 600, 64


def both(up, across):
    """The weights and a place for their gradient, so many rows and columns on, in one buffer."""
    h, w, t, grad = make(21, ROWS, VOCAB, K)
    buf = torch.zeros(2 * VOCAB, 2 * K, device="cuda", dtype=torch.bfloat16)
    weight, d_weight = buf[:VOCAB, :K], buf[up:VOCAB + up, across:K + across]
    weight.copy_(w)
    return h, weight, t, grad, d_weight


@pytest.mark.parametrize("up,across", [(0, 0), (1, 0), (VOCAB - 1, 0), (0, 1), (5, K - 1)])
def test_refused(monkeypatch, up, across):
    def enqueued(*args, **kw):
        raise AssertionError("the call went on")
    h, w, t, grad, dw = both(up, across)
    lse = torch.zeros(ROWS, device="cuda")
    monkeypatch.setattr(B, "reflex_head_loss_backward", enqueued)
    with pytest.raises(ValueError):
        api.head_loss_backward(h, w, t, lse, grad, d_weight=dw)


@pytest.mark.parametrize("up,across", [(0, K), (VOCAB, 0), (VOCAB, K), (1, K)])
def test_beside_the_weights(up, across):
    h, w, t, grad, dw = both(up, across)
    kept = w.clone()
    loss, lse = api.head_loss(h, w, t)
    dh, got = api.head_loss_backward(h, w, t, lse, grad, d_weight=dw)
    assert got is dw and torch.equal(w, kept)
    check_grad(h, w, t, grad, dh, dw)


def test_gradients_of_the_rows_refused(monkeypatch):
    def enqueued(*args, **kw):
        raise AssertionError("the call went on")
    h, w, t, grad, dw = both(VOCAB, 0)
    lse = torch.zeros(ROWS, device="cuda")
    monkeypatch.setattr(B, "reflex_head_loss_backward", enqueued)
    for kw in (dict(d_hidden=w[:ROWS]), dict(d_hidden=w[VOCAB - ROWS:], need_weight=False),
               dict(d_hidden=dw[7:7 + ROWS], d_weight=dw)):
        with pytest.raises(ValueError):
            api.head_loss_backward(h, w, t, lse, grad, **kw)
