"""The weights' gradient of banned tokens (a logit of -inf): G is 0 there, in rows that
count as in those that only fill a tile, and so is the gradient of the token's weights."""
import pytest
import torch

from test_gpu_head_loss_banned import BANNED, banned
from paper_2608_01784_gb300 import api

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows", [1, 40, 64, 65, 300, 512])
def test_gradient_of_the_weights(rows, dtype):
    got = []
    for lowest in (-float("inf"), -2.0 ** 100):
        h, w, t, grad = banned(rows, 64, lowest=lowest)
        loss, lse = api.head_loss(h, w, t)
        dw = torch.full(w.shape, 7.0, device="cuda", dtype=dtype)
        api.head_loss_backward(h, w, t, lse, grad, d_weight=dw, need_hidden=False)
        got.append(dw)
    assert torch.equal(*got) and not got[0][BANNED].any() and bool(got[0].isfinite().all())
