"""Rows next to the largest fp32 value times small weights: the product is finite and
so is every sum on the way, whichever kernel the number of rows picks."""
import pytest
import torch

from paper_2608_01784_gb300 import _binding as B
from paper_2608_01784_gb300 import api
from tests.test_gpu_fp8 import (BF16, F32, check_experts, check_product, codes_of, experts64,
                                normal, product_bound, routing)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,k", [(5, 77), (130, 512), (64, 2048)])
@pytest.mark.parametrize("size", [1e34, 1e36, 5e37])
def test_linear_of_large_rows(n, k, dtype, size):
    w, ws = api.quantize_fp8(normal(n, n, k, std=1e-12), 128)
    x = (normal(k, 6, k) * size).clamp(-3.3e38, 3.3e38).to(dtype)
    x[1] *= 1e-6   # large and small blocks in one row
    x[2, : k // 2] *= 1e-30
    codes, scales = codes_of(x, 1)
    ref, bound = product_bound(codes.cuda(), scales.cuda(), w, ws)
    lin = api.LinearFp8(w, ws, max_rows=6, out_dtype=F32)
    for m in range(1, 7):
        check_product(lin.forward(x[:m]), ref[:m], bound[:m], True)


# two slots a token: a few pairs in two launches, and tiles
@pytest.mark.parametrize("T", [1, 3, 70])
@pytest.mark.parametrize("h_std,up_std,down_std", [
    (1e37, 1e-28, 1e-15),   # large rows
    (1e9, 2e8, 1e-20)])     # large activations
def test_experts_of_large_rows(T, h_std, up_std, down_std):
    d, E, inter, k_max = 64, 6, 128, 2
    w = api.quantize_experts(normal(1, E, 2 * inter, d, std=up_std),
                             normal(2, E, d, inter, std=down_std))
    h = (normal(T, T, d) * h_std).to(BF16)
    ids, alpha, k = routing(T, T, E, k_max)
    op = api.ExpertsFp8(w, d=d, E=E, inter=inter, k_max=k_max, max_tokens=T)
    out = op.forward(h, ids, alpha, k)
    assert op.status() == B.REFLEX_OK
    check_experts(out, experts64(h, ids, alpha, w, inter))
