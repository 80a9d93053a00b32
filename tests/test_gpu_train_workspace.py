"""No call around the experts writes behind the workspace that it asks for."""
import pytest
import torch

from test_gpu_head_loss import check_grad, check_loss, make
from paper_2608_01784_gb300 import _binding as B

pytestmark = pytest.mark.gpu
GUARD = 1 << 20


def guarded(nbytes):
    return torch.full((nbytes + GUARD,), 0x5A, dtype=torch.uint8, device="cuda")


def whole(ws, nbytes):
    return bool((ws[nbytes:] == 0x5A).all())


@pytest.mark.parametrize("vocab", [1, 9, 17, 150, 153, 1000, 2000, 2400, 4500, 4700, 20000])
@pytest.mark.parametrize("rows", [1, 31, 32, 33, 64, 65, 300])
def test_head_loss(rows, vocab):
    k = 72
    h, w, t, grad = make(rows + vocab, rows, vocab, k, 0.9)
    loss, lse = (torch.full((rows,), 7.0, device="cuda") for _ in range(2))
    n = B.reflex_head_loss_workspace_size(rows, vocab, k)
    ws = guarded(n)
    B.reflex_head_loss(h, k, w, k, t, rows, vocab, k, loss, lse, None, ws, n, None)
    assert whole(ws, n)
    check_loss(h, w, t, loss, lse)
    n = B.reflex_head_loss_backward_workspace_size(rows, vocab, k)
    ws = guarded(n)
    dh, dw = torch.empty_like(h), torch.empty(vocab, k, dtype=h.dtype, device="cuda")
    B.reflex_head_loss_backward(h, k, w, k, t, lse, grad, rows, vocab, k, B.REFLEX_DTYPE_BF16, dh, k,
                                B.REFLEX_DTYPE_BF16, dw, k, None, ws, n, None)
    assert whole(ws, n)
    check_grad(h, w, t, grad, dh, dw)


@pytest.mark.parametrize("rows,d", [(1, 1), (3, 7), (700, 100), (5000, 31), (2000, 1001),
                                    (1300, 2048), (40, 16384)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_block_norm(rows, d, dtype):
    h, y, do, dn, dh, dy = (torch.randn(rows, d, device="cuda").to(dtype) for _ in range(6))
    w1, w2, gate, dw1, dw2, dg = (torch.ones(d, device="cuda", dtype=dtype) for _ in range(6))
    n = B.reflex_block_norm_workspace_size(rows, d)
    ws = guarded(n)
    code = B.REFLEX_DTYPE_F32 if dtype == torch.float32 else B.REFLEX_DTYPE_BF16
    B.reflex_block_norm_backward(code, h, d, y, d, w1, gate, 0, w2, 1.0, 1e-6, rows, d, do, d, dn, d,
                                 dh, d, dy, d, dg, d, dw1, dw2, ws, n, None)
    assert whole(ws, n)


@pytest.mark.parametrize("T,E,k_max", [(0, 8, 4), (1, 1, 1), (300, 64, 12), (32768, 64, 12),
                                       (5000, 1024, 32), (100001, 7, 3)])
def test_expert_plan(T, E, k_max):
    ids = torch.randint(0, E, (T, k_max), device="cuda", dtype=torch.int32)
    row_of, counts, offsets = (torch.full((m + 64,), 77, device="cuda", dtype=torch.int32)
                               for m in (T * k_max, E, E + 1))
    n = B.reflex_expert_plan_workspace_size(T, E, k_max)
    ws = guarded(n)
    B.reflex_expert_plan(ids, None, T, E, k_max, T * k_max, row_of, counts, offsets, None, None, ws, n,
                         None)
    assert whole(ws, n)
    assert all(bool((x[-64:] == 77).all()) for x in (row_of, counts, offsets))
    assert int(offsets[E]) == T * k_max
