"""The 8-bit products where their kernels change over: few rows, split K, edges of
the boxes that tiles are stored in, groups around them, rows far apart."""
import pytest
import torch

from paper_2608_01784_gb300 import _binding as B
from paper_2608_01784_gb300 import api
from tests.test_gpu_fp8 import (BF16, E4M3, F32, check_experts, check_product, codes_of, experts64,
                                experts_layer, normal, product_bound, routing, same_codes)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,out_dtype", [(F32, BF16), (BF16, F32)])
@pytest.mark.parametrize("n", [1, 3, 5, 130])
@pytest.mark.parametrize("k", [1, 15, 16, 511, 513, 2048, 4100, 16384, 16400])
def test_few_rows(n, k, dtype, out_dtype):
    w, ws = api.quantize_fp8(normal(n + k, n, k, std=0.02), 128)
    x = normal(k, 5, k, dtype=dtype)
    codes, scales = codes_of(x, 1)
    ref, bound = product_bound(codes.cuda(), scales.cuda(), w, ws)
    lin = api.LinearFp8(w, ws, max_rows=5)
    whole = torch.full((5, n + 1), 7.0, dtype=out_dtype, device="cuda")  # rows off 4 bytes
    for m in range(1, 6):
        lin.forward(x[:m], out=whole[:m, 1:])
        check_product(whole[:m, 1:], ref[:m], bound[:m], out_dtype == F32)
        assert bool((whole[:, 0] == 7.0).all()) and bool((whole[m:] == 7.0).all())
        assert lin.status() == B.REFLEX_OK


@pytest.mark.parametrize("m", [1, 31, 32, 33, 128, 129, 161, 256])
@pytest.mark.parametrize("n", [8, 63, 64, 72, 130, 200, 257, 264])
def test_edges_of_stored_boxes(m, n):
    """bf16 rows on 16-byte boundaries: nothing outside [m, n] is written."""
    k = 200
    a, sa = api.quantize_fp8(normal(m, m, k))
    b, sb = api.quantize_fp8(normal(n, n, k, std=0.05), 128)
    whole = torch.full((m + 40, -(-n // 8) * 8 + 16), 7.0, dtype=BF16, device="cuda")
    out = api.matmul_fp8(a, sa, b, sb, out=whole[2:m + 2, 8:n + 8])
    check_product(out, *product_bound(a, sa, b, sb), False)
    out.fill_(7.0)
    assert bool((whole == 7.0).all())


@pytest.mark.parametrize("m,n,k", [(8, 1024, 8192), (33, 256, 8300), (128, 1000, 8192),
                                   (300, 300, 8320), (5, 5000, 1024), (32, 777, 1500)])
@pytest.mark.parametrize("out_dtype", [F32, BF16])
def test_shared_tiles_of_long_rows(m, n, k, out_dtype):
    a, sa = api.quantize_fp8(normal(m, m, k))
    b, sb = api.quantize_fp8(normal(n, n, k, std=0.05), 128)
    ref, bound = product_bound(a, sa, b, sb)
    whole = torch.full((m, n + 3), 7.0, dtype=out_dtype, device="cuda")
    check_product(api.matmul_fp8(a, sa, b, sb, out=whole[:, :n]), ref, bound, out_dtype == F32)
    assert bool((whole[:, n:] == 7.0).all())
    out = api.matmul_fp8(a, sa, b, sb, out_dtype=out_dtype)
    check_product(out, ref, bound, out_dtype == F32)
    assert torch.equal(out, whole[:, :n])


@pytest.mark.parametrize("n", [7, 31, 33, 5001])
@pytest.mark.parametrize("out_dtype", [F32, BF16])
def test_new_outputs_have_aligned_rows(n, out_dtype):
    w, ws = api.quantize_fp8(normal(n, n, 300, std=0.05), 128)
    x = normal(1, 40, 300, dtype=BF16)
    lin = api.LinearFp8(w, ws, max_rows=40, out_dtype=out_dtype)
    out = lin.forward(x)
    assert out.shape == (40, n) and out.dtype == out_dtype
    unit = 16 // out.element_size()
    assert out.stride(0) % unit == 0 if n >= 4 * unit else out.stride(0) == n
    packed = torch.empty((40, n), dtype=out_dtype, device="cuda")
    assert torch.equal(lin.forward(x, packed), out)


@pytest.mark.parametrize("inter", [64, 192, 256])
def test_groups_of_any_size(inter):
    """Pairs of an expert just below, at and above the stored boxes and the tiles."""
    sizes = [0, 1, 31, 32, 33, 63, 64, 65, 127, 0, 128, 129, 159, 160, 161, 255, 256, 257, 300, 0]
    E, d = len(sizes), 256
    ids = torch.repeat_interleave(torch.arange(E), torch.tensor(sizes)).int()
    T = ids.numel()
    ids = ids[torch.randperm(T, generator=torch.Generator().manual_seed(inter))].cuda()[:, None]
    alpha = normal(3, T, 1).abs()
    k = torch.ones(T, dtype=torch.int32, device="cuda")
    w = experts_layer(inter, d, E, inter)
    h = normal(4, T, d, dtype=BF16)
    op = api.ExpertsFp8(w, d=d, E=E, inter=inter, k_max=1, max_tokens=T)
    out = op.forward(h, ids.contiguous(), alpha, k)
    assert op.status() == B.REFLEX_OK
    check_experts(out, experts64(h, ids, alpha, w, inter))


def far(rows, cols, dtype):
    """Rows further apart than 32 bits of bytes reach."""
    ld = (1 << 31) // torch.empty((), dtype=dtype).element_size() + 16
    return torch.empty(rows * ld, dtype=dtype, device="cuda").as_strided((rows, cols), (ld, 1))


def test_rows_far_apart():
    m, n, k = 3, 300, 200
    x = far(m, k, BF16)
    x.copy_(normal(1, m, k))
    a, sa = api.quantize_fp8(x, 1, far(m, k, E4M3), far(m, 2, F32))
    want, scales = api.quantize_fp8(x.contiguous())
    assert same_codes(a, want) and torch.equal(sa, scales)
    b, sb = api.quantize_fp8(normal(2, n, k, std=0.05), 128)
    ref, bound = product_bound(want, scales, b, sb)
    for out_dtype in (F32, BF16):
        check_product(api.matmul_fp8(a, sa, b, sb, out=far(m, n, out_dtype)), ref, bound,
                      out_dtype == F32)
    lin = api.LinearFp8(b, sb, max_rows=m)
    check_product(lin.forward(x, far(m, n, BF16)), ref, bound, False)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_logits_far_apart(dtype):
    z = far(3, 1000, dtype)
    z.copy_(normal(5, 3, 1000, std=3.0))
    u = torch.tensor([0.1, 0.5, 0.9], device="cuda")
    top = torch.full((3,), 40, dtype=torch.int32, device="cuda")
    for kw in ({}, dict(top_k=top)):
        got, want = api.sample(z, u, **kw), api.sample(z.contiguous(), u, **kw)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("m,n,k", [(3, 40, 100), (2, 300, 17), (40, 300, 1000), (200, 130, 77),
                                   (33, 64, 8201)])
def test_what_follows_a_row_is_not_read(m, n, k):
    """NaN codes between the rows of A and B, and in a workspace used before."""
    def spread(codes):
        wide = torch.full((codes.shape[0], -(-k // 16) * 16 + 16), 0x7f, dtype=torch.uint8,
                          device="cuda")
        wide[:, :k] = codes.view(torch.uint8)
        return wide.view(E4M3)[:, :k]
    x = normal(m, m, k)
    a, sa = api.quantize_fp8(x)
    b, sb = api.quantize_fp8(normal(n, n, k, std=0.05), 128)
    ref, bound = product_bound(a, sa, b, sb)
    wide = spread(b)
    check_product(api.matmul_fp8(spread(a), sa, wide, sb, out_dtype=F32), ref, bound, True)
    lin = api.LinearFp8(wide, sb, max_rows=m, out_dtype=F32)
    lin.ws.fill_(0x7f)
    check_product(lin.forward(x), ref, bound, True)
    assert lin.status() == B.REFLEX_OK


@pytest.mark.parametrize("T,d,E,inter,k_max", [(1, 64, 4, 64, 2), (70, 320, 6, 192, 4),
                                               (900, 256, 5, 128, 3)])
def test_experts_whatever_the_workspace_holds(T, d, E, inter, k_max):
    w = experts_layer(T, d, E, inter)
    h = normal(2, T, d, dtype=BF16)
    ids, alpha, k = routing(T, T, E, k_max)
    op = api.ExpertsFp8(w, d=d, E=E, inter=inter, k_max=k_max, max_tokens=T)
    outs = []
    for byte in (0x00, 0x7f, 0xff):
        op.ws.fill_(byte)
        outs.append(op.forward(h, ids, alpha, k))
        assert op.status() == B.REFLEX_OK
    check_experts(outs[0], experts64(h, ids, alpha, w, inter))
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


@pytest.mark.parametrize("T,d,inter,k_max", [
    (64, 128, 64, 2), (65, 128, 64, 2),            # 128 and 130 slots
    (4, 2048, 1024, 6), (5, 2048, 1024, 6),        # 151 and 189 MB of the slots' weights
    (1, 576, 320, 32), (3, 64, 64, 32), (2, 4096, 192, 3), (1, 640, 4160, 2)])
def test_few_pairs_and_more(T, d, inter, k_max):
    """Around the sizes from which tiles of the tensor cores take over."""
    E = 40
    w = experts_layer(T + d, d, E, inter)
    h = normal(T, T, d, dtype=BF16)
    ids, alpha, k = routing(T + E, T, E, k_max)
    op = api.ExpertsFp8(w, d=d, E=E, inter=inter, k_max=k_max, max_tokens=T)
    out = op.forward(h, ids, alpha, k)
    assert op.status() == B.REFLEX_OK
    ref = experts64(h, ids, alpha, w, inter)
    check_experts(out, ref)
    assert torch.equal(op.forward(h, ids, alpha, k), out)
    both = op.forward(h, ids, alpha, k, residual=True).double() - (h.double() + ref)
    assert float(both.norm() / (h.double() + ref).norm()) <= 6e-3


@pytest.mark.parametrize("T", [7, 200])
def test_experts_errors_and_nan(T):
    d, E, inter, k_max = 192, 4, 128, 2
    w = experts_layer(4, d, E, inter)
    op = api.ExpertsFp8(w, d=d, E=E, inter=inter, k_max=k_max, max_tokens=T)
    h = normal(1, T, d, dtype=BF16)
    ids, alpha, k = routing(1, T, E, k_max, lo=2)
    want = op.forward(h, ids, alpha, k)
    rest = torch.arange(T, device="cuda") != 3
    for bad in (E, -7):
        wrong = ids.clone()
        wrong[3, 1] = bad
        out = op.forward(h, wrong, alpha, k)
        assert op.status() == B.REFLEX_EINVAL and torch.equal(out[rest], want[rest])
        only = alpha.clone()
        only[3, 1] = 0.0
        check_experts(out, experts64(h, ids, only, w, inter))
    for count, same in ((3, 2), (0, 1), (-5, 1)):
        counts = k.clone()
        counts[3] = count
        out = op.forward(h, ids, alpha, counts)
        assert op.status() == B.REFLEX_EKRANGE and torch.equal(out[rest], want[rest])
        counts[3] = same
        assert torch.equal(out, op.forward(h, ids, alpha, counts)) and op.status() == B.REFLEX_OK
    h[3, 5] = float("nan")
    out = op.forward(h, ids, alpha, k)
    assert bool(out[3].isnan().all()) and torch.equal(out[rest], want[rest])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols,extra", [(1001, 1, 0), (77, 100, 4), (3, 128, 0), (123, 300, 1),
                                             (9, 512, 8), (10, 513, 0), (70001, 129, 0),
                                             (5, 1025, 7)])
def test_narrow_and_wide_rows_quantised(rows, cols, extra, dtype):
    x = torch.full((rows, cols + extra), float("nan"), dtype=dtype, device="cuda")
    x[:, :cols] = normal(rows + cols, rows, cols)
    whole = torch.full((rows + 1, cols + 3), 0x55, dtype=torch.uint8, device="cuda")
    codes, scales = api.quantize_fp8(x[:, :cols], 1, whole.view(E4M3)[:rows, :cols])
    want, want_scales = codes_of(x[:, :cols], 1)
    assert same_codes(codes, want) and torch.equal(scales.cpu(), want_scales)
    assert bool((whole[:, cols:] == 0x55).all()) and bool((whole[rows:] == 0x55).all())
