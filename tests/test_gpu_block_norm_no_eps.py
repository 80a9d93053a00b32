"""Gradients of norms with eps = 0: rows of zeros that only fill a warp stay out of the
weights' sums (bounds: test_gpu_block_norm)."""
import pytest
import torch

from test_gpu_block_norm import check_backward, check_forward, make
from paper_2608_01784_gb300 import api

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("gate", ["none", "channel", "token"])
@pytest.mark.parametrize("rows,d", [(1, 8), (3, 8), (5, 31), (13, 16), (1, 100), (7, 100), (9, 128),
                                    (300, 64), (4001, 24), (3, 200), (2, 1000)])
def test_no_eps(rows, d, gate, dtype):
    h, y, opt, d_out, d_norm = make(rows * 7 + d, rows, d, dtype, gate=gate)
    opt["eps"] = 0.0
    check_forward(h, y, opt, *api.block_norm(h, y, **opt))
    check_backward(h, y, opt, d_out, d_norm, api.block_norm_backward(h, y, d_out, d_norm, **opt))


@pytest.mark.parametrize("rows,d", [(3, 8), (7, 100)])
def test_a_norm_alone(rows, d):
    h, _, opt, _, d_norm = make(rows, rows, d, torch.float32, after=False, gate="none")
    opt["eps"] = 0.0
    check_backward(h, None, opt, None, d_norm, api.block_norm_backward(h, None, None, d_norm, **opt))
