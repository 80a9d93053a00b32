"""The 8-bit products on the GPU against their formulas in 64 bits: codes and
scales bit for bit, products within the bound of their fp32 sums, routed experts
within the rounding of what they store."""
import numpy as np
import pytest
import torch

from paper_2608_01784_gb300 import _binding as B
from paper_2608_01784_gb300 import api

pytestmark = pytest.mark.gpu

BF16, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


def blocks(n):
    return -(-n // 128)


def normal(seed, *shape, std=1.0, dtype=F32):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * std).to(dtype).cuda()


def strided(t, extra):
    """The same matrix with `extra` more elements between its rows."""
    r, c = t.shape
    w = torch.full((r, c + extra), float("nan"), dtype=t.dtype, device=t.device)
    w[:, :c] = t
    return w[:, :c]


def codes_of(x, block_rows):
    """Codes and scales by the formula's fp32 operations, on the host."""
    x = x.float().cpu()
    r, c = x.shape
    p = torch.zeros(-(-r // block_rows) * block_rows, blocks(c) * 128)
    p[:r, :c] = x
    p = p.view(-1, block_rows, blocks(c), 128)
    a = p.abs().amax((1, 3), keepdim=True).clamp(min=2.0 ** -100)
    codes = (p * (a.reciprocal() * 448.0)).to(E4M3).view(-1, blocks(c) * 128)
    return codes[:r, :c], (a / 448.0)[:, 0, :, 0]


def same_codes(a, b):
    return torch.equal(torch.nan_to_num(a.float().cpu(), nan=1e9),
                       torch.nan_to_num(b.float().cpu(), nan=1e9))


def values(codes, scales, block_rows=1):
    r, c = codes.shape
    at = torch.arange(r, device=codes.device) // block_rows
    return codes.double() * scales.double()[at][:, torch.arange(c, device=codes.device) // 128]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("rows,cols,extra", [
    (1, 1, 0), (1, 2048, 0), (5, 127, 0), (130, 129, 0), (33, 1000, 24), (257, 513, 3),
    (700, 2048, 8), (1, 16, 1), (2000, 5, 0)])
def test_quantize_bits(dtype, block_rows, rows, cols, extra):
    x = normal(rows * 7 + cols, rows, cols, dtype=dtype)
    x *= torch.exp2(torch.arange(rows, device="cuda") % 40 - 20)[:, None].to(dtype)
    x = strided(x, extra) if extra else x
    codes, scales = api.quantize_fp8(x, block_rows)
    want_c, want_s = codes_of(x, block_rows)
    assert torch.equal(scales.cpu(), want_s)
    assert same_codes(codes, want_c)
    # half a step of e4m3 (2^-4 of a normal value, 2^-10 of the scale below), the
    # fp32 roundings of the scale and of the product on top
    err = (values(codes, scales, block_rows) - x.double()).abs()
    at = torch.arange(rows, device="cuda") // block_rows
    s = scales.double()[at][:, torch.arange(cols, device="cuda") // 128]
    assert bool((err <= (x.double().abs() * 2.0 ** -4).maximum(s * 2.0 ** -10) * (1 + 2e-6) +
                 2e-7 * x.double().abs()).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_quantize_special_values(dtype):
    x = torch.ones(8, 300, dtype=dtype)
    x[0] = 0
    x[1, 5] = float("inf")
    x[2, 130] = float("nan")
    x[3] = -0.0
    x[4] = 1e-38
    x[5] = 3e38
    x[6, 299] = -float("inf")
    x[7] = 1e-30
    x = x.cuda()
    codes, scales = api.quantize_fp8(x)
    want_c, want_s = codes_of(x, 1)
    assert torch.equal(torch.nan_to_num(scales.cpu(), nan=-1.0), torch.nan_to_num(want_s, nan=-1.0))
    assert same_codes(codes, want_c)
    v = values(codes, scales)
    assert bool((v[0] == 0).all()) and bool((v[3] == 0).all())
    assert bool(v[1, :128].isnan().all()) and bool(((v[1, 128:] - 1).abs() <= 2.0 ** -23).all())
    assert bool(v[2, 128:256].isnan().all()) and not bool(v[2, :128].isnan().any())
    assert bool(v[6, 256:].isnan().all())


def test_quantize_nothing_and_refusals():
    c, s = api.quantize_fp8(torch.empty(0, 64, device="cuda"))
    assert c.shape == (0, 64) and s.shape == (0, 1)
    x = torch.zeros(4, 64, device="cuda")
    with pytest.raises(ValueError):
        api.quantize_fp8(x, 64)
    with pytest.raises(ValueError):
        api.quantize_fp8(x.t())
    with pytest.raises(ValueError):
        api.quantize_fp8(x.half())
    with pytest.raises(ValueError):
        api.quantize_fp8(x, codes=torch.empty(4, 32, dtype=E4M3, device="cuda"))


def product_bound(a, sa, b, sb):
    """What the sums may be off: products of codes are exact, a block of 128 is
    summed in fp32 (each addition rounded or cut, 2^-23), scaled (2 roundings)
    and added to the others; relative to the sum of magnitudes."""
    va, vb = values(a, sa), values(b, sb, 128)
    ref = va @ vb.T
    mag = va.abs() @ vb.abs().T
    return ref, mag * (128 + 2 * blocks(a.shape[1]) + 4) * 2.0 ** -23


def check_product(out, ref, bound, f32):
    tol = bound + (0 if f32 else ref.abs() * 2.0 ** -8) + 1e-37
    err = (out.double() - ref).abs()
    assert bool((err <= tol).all()), float((err / tol).max())


SHAPES = [  # rows, columns, K: single tokens, splits of K, odd sizes, several tiles
    (1, 1, 1), (1, 4096, 2048), (2, 256, 128), (7, 300, 100), (31, 257, 4096), (32, 128, 256),
    (33, 129, 640), (64, 2048, 2048), (127, 1000, 1111), (128, 256, 512), (129, 255, 384),
    (200, 513, 1029), (300, 5000, 256), (1000, 777, 2048), (4000, 640, 128), (520, 4100, 1024)]


@pytest.mark.parametrize("out_dtype", [F32, BF16])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_matmul(m, n, k, out_dtype):
    a, sa = api.quantize_fp8(normal(m + n + k, m, k))
    b, sb = api.quantize_fp8(normal(m * n + k, n, k, std=0.02), 128)
    status = torch.full((1,), 99, dtype=torch.int32, device="cuda")
    out = api.matmul_fp8(a, sa, b, sb, out_dtype=out_dtype, status=status)
    ref, bound = product_bound(a, sa, b, sb)
    check_product(out, ref, bound, out_dtype == F32)
    assert B.reflex_read_status(status) == B.REFLEX_OK
    assert torch.equal(out, api.matmul_fp8(a, sa, b, sb, out_dtype=out_dtype))


@pytest.mark.parametrize("m,n,k", [(3, 100, 300), (140, 270, 256), (40, 1024, 2048)])
@pytest.mark.parametrize("out_dtype", [F32, BF16])
@pytest.mark.parametrize("extra", [1, 8])
def test_matmul_strides(m, n, k, out_dtype, extra):
    """Rows of out at any stride; what lies between them stays."""
    a, sa = api.quantize_fp8(normal(1, m, k))
    b, sb = api.quantize_fp8(normal(2, n, k), 128)
    whole = torch.full((m, n + extra), 7.0, dtype=out_dtype, device="cuda")
    sa, sb = strided(sa, 3), strided(sb, 2)
    a2 = torch.empty((m, -(-k // 16) * 16 + 32), dtype=E4M3, device="cuda")[:, :k]
    a2.view(torch.uint8).copy_(a.view(torch.uint8))
    out = api.matmul_fp8(a2, sa, b, sb, out=whole[:, :n])
    ref, bound = product_bound(a, sa, b, sb)
    check_product(out, ref, bound, out_dtype == F32)
    assert bool((whole[:, n:] == 7.0).all())


def test_matmul_scales_of_any_size():
    """Blocks of very different scales: each is scaled by itself, in fp32."""
    m, n, k = 70, 300, 1024
    a, sa = api.quantize_fp8(normal(5, m, k))
    b, sb = api.quantize_fp8(normal(6, n, k), 128)
    g = torch.Generator().manual_seed(3)
    sa = sa * torch.exp2(torch.randint(-30, 30, sa.shape, generator=g).float()).cuda()
    sb = sb * torch.exp2(torch.randint(-30, 30, sb.shape, generator=g).float()).cuda()
    ref, bound = product_bound(a, sa, b, sb)
    check_product(api.matmul_fp8(a, sa, b, sb, out_dtype=F32), ref, bound, True)


def test_matmul_nan_stays_in_its_row_and_column():
    m, n, k = 40, 300, 512
    a, sa = api.quantize_fp8(normal(8, m, k))
    b, sb = api.quantize_fp8(normal(9, n, k), 128)
    sa[17, 2] = float("nan")
    out = api.matmul_fp8(a, sa, b, sb, out_dtype=F32)
    assert bool(out[17].isnan().all()) and not bool(out[torch.arange(m) != 17].isnan().any())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m,n,k", [(1, 4096, 2048), (3, 50, 77), (32, 5001, 1000), (260, 512, 2048)])
def test_linear(dtype, m, n, k):
    x = normal(m + 3, m, k, dtype=dtype)
    w, ws = api.quantize_fp8(normal(n, n, k, std=0.02), 128)
    lin = api.LinearFp8(w, ws, max_rows=m + 5, out_dtype=F32)
    out = lin.forward(x)
    codes, scales = codes_of(x, 1)
    ref, bound = product_bound(codes.cuda(), scales.cuda(), w, ws)
    check_product(out, ref, bound, True)
    assert lin.status() == B.REFLEX_OK
    wide = strided(x, 5)
    assert torch.equal(lin.forward(wide), out)
    assert lin.forward(x[:0]).shape == (0, n)
    # fewer rows: another number of CTAs may share K
    if m > 1:
        check_product(lin.forward(x[:1]), ref[:1], bound[:1], True)


def test_linear_on_another_stream_and_in_a_graph():
    x = normal(1, 48, 1024, dtype=BF16)
    w, ws = api.quantize_fp8(normal(2, 2000, 1024, std=0.02), 128)
    lin = api.LinearFp8(w, ws, max_rows=48)
    want = lin.forward(x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = lin.forward(x)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got, want)
    out = torch.empty_like(want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        lin.forward(x, out)
    x.copy_(normal(7, 48, 1024, dtype=BF16))
    g.replay()
    again = lin.forward(x)
    assert torch.equal(out, again) and not torch.equal(out, want)


def test_linear_refusals():
    w, ws = api.quantize_fp8(normal(2, 200, 256), 128)
    lin = api.LinearFp8(w, ws, max_rows=4)
    for bad in (normal(1, 5, 256), normal(1, 4, 128), normal(1, 4, 256).half(),
                normal(1, 256, 4).t(), normal(1, 4, 256).cpu()):
        with pytest.raises(ValueError):
            lin.forward(bad)
    with pytest.raises(ValueError):
        api.LinearFp8(w[:, 1:], ws, max_rows=4)
    with pytest.raises(ValueError):
        api.LinearFp8(w, ws[:1], max_rows=4)
    with pytest.raises(ValueError):
        api.matmul_fp8(w, torch.ones(200, 3, device="cuda"), w, ws)


def routing(seed, T, E, k_max, lo=1, skew=0.0):
    g = torch.Generator().manual_seed(seed)
    most = min(k_max, E)
    z = torch.randn(T, E, generator=g) + skew * torch.arange(E, 0, -1)
    k = torch.randint(min(lo, most), most + 1, (T,), generator=g, dtype=torch.int32)
    top = torch.topk(z, most, dim=1)
    used = torch.arange(k_max)[None] < k[:, None]
    ids = torch.full((T, k_max), -1, dtype=torch.int32)
    ids[:, :most] = top.indices.int()
    alpha = torch.zeros(T, k_max)
    alpha[:, :most] = torch.softmax(top.values.masked_fill(~used[:, :most], -1e30), 1)
    return torch.where(used, ids, -1).cuda(), (alpha * used).cuda(), k.cuda()


def experts64(h, ids, alpha, w, inter):
    """The layer in 64 bits on the same codes; the activation's codes by the formula."""
    c, s = codes_of(h, 1)
    x = values(c.cuda(), s.cuda())
    out = torch.zeros_like(x)
    for e in range(w["w_down"].shape[0]):
        t, j = torch.nonzero(ids == e, as_tuple=True)
        if not t.numel():
            continue
        gu, gus = w["w_gate_up"][e], w["w_gate_up_scales"][e]
        g = x[t] @ values(gu[:inter], gus[0], 128).T
        a = g * torch.sigmoid(g) * (x[t] @ values(gu[inter:], gus[1], 128).T)
        ac, as_ = codes_of(a, 1)
        y = values(ac.cuda(), as_.cuda()) @ values(w["w_down"][e], w["w_down_scales"][e], 128).T
        out.index_add_(0, t, alpha[t, j].double()[:, None] * y)
    return out


def experts_layer(seed, d, E, inter):
    return api.quantize_experts(normal(seed, E, 2 * inter, d, std=0.05),
                                normal(seed + 1, E, d, inter, std=0.05))


def check_experts(out, ref):
    # bf16 pair outputs and a bf16 sum: 2^-9 each of the largest terms (2e-3 rms);
    # an activation next to the middle of two codes may take the other one, 6% of
    # one of `inter` terms.  Relative to the output's rms: a few roundings, one element
    # a few standard deviations of that.
    err, rms = (out.double() - ref), ref.square().mean().sqrt()
    assert float(err.square().mean().sqrt() / rms) <= 6e-3
    assert float((err.abs() / ref.abs().maximum(rms)).max()) <= 0.1


@pytest.mark.parametrize("T,d,E,inter,k_max,skew", [
    (1, 256, 8, 128, 4, 0.0), (1, 2048, 64, 1024, 12, 0.0), (5, 64, 3, 64, 4, 0.0),
    (32, 512, 16, 256, 8, 0.0), (33, 320, 12, 192, 12, 0.0), (100, 256, 5, 576, 5, 1.0),
    (300, 1024, 8, 512, 2, 2.0), (1000, 512, 60, 128, 8, 0.05), (700, 256, 1, 128, 1, 0.0),
    (96, 4096, 32, 128, 12, 0.3), (4200, 128, 40, 64, 6, 0.1), (64, 256, 300, 128, 8, 0.0),
    (50, 192, 1024, 64, 32, 0.0)])
def test_experts(T, d, E, inter, k_max, skew):
    w = experts_layer(T + d, d, E, inter)
    h = normal(T, T, d, dtype=BF16)
    ids, alpha, k = routing(T + E, T, E, k_max, skew=skew)
    op = api.ExpertsFp8(w, d=d, E=E, inter=inter, k_max=k_max, max_tokens=T + 3)
    out = op.forward(h, ids, alpha, k)
    assert op.status() == B.REFLEX_OK
    ref = experts64(h, ids, alpha, w, inter)
    check_experts(out, ref)
    assert torch.equal(op.forward(h, ids, alpha, k), out)
    res = op.forward(h, ids, alpha, k, residual=True)
    both = h.double() + ref
    assert float((res.double() - both).norm() / both.norm()) <= 6e-3


def test_experts_rows_of_few_tokens_in_a_large_workspace():
    """A workspace sized for many tokens serves few; nothing of an earlier call is left."""
    d, E, inter, k_max = 256, 16, 128, 4
    w = experts_layer(3, d, E, inter)
    op = api.ExpertsFp8(w, d=d, E=E, inter=inter, k_max=k_max, max_tokens=5000)
    for T in (5000, 3, 129, 1, 0):
        h = normal(T, T, d, dtype=BF16)
        ids, alpha, k = routing(T, T, E, k_max)
        out = op.forward(h, ids, alpha, k)
        assert op.status() == B.REFLEX_OK
        if T:
            check_experts(out, experts64(h, ids, alpha, w, inter))


def test_experts_device_errors():
    d, E, inter, k_max = 128, 4, 64, 2
    w = experts_layer(4, d, E, inter)
    op = api.ExpertsFp8(w, d=d, E=E, inter=inter, k_max=k_max, max_tokens=40)
    h = normal(1, 40, d, dtype=BF16)
    ids, alpha, k = routing(1, 40, E, k_max, lo=2)
    want = op.forward(h, ids, alpha, k)
    bad = ids.clone()
    bad[3, 0], bad[5, 1] = E, -7
    out = op.forward(h, bad, alpha, k)
    assert op.status() == B.REFLEX_EINVAL
    rest = torch.tensor([t for t in range(40) if t not in (3, 5)])
    assert torch.equal(out[rest], want[rest])
    many = k.clone()
    many[7] = 3
    op.forward(h, ids, alpha, many)
    assert op.status() == B.REFLEX_EKRANGE
    op.forward(h, ids, alpha, k)
    assert op.status() == B.REFLEX_OK


def test_experts_nan_stays_in_its_token():
    d, E, inter, k_max = 256, 4, 128, 2
    w = experts_layer(5, d, E, inter)
    op = api.ExpertsFp8(w, d=d, E=E, inter=inter, k_max=k_max, max_tokens=200)
    h = normal(1, 200, d, dtype=BF16)
    ids, alpha, k = routing(1, 200, E, k_max)
    want = op.forward(h, ids, alpha, k)
    h[11, 40] = float("nan")
    h[90, 7] = float("inf")
    out = op.forward(h, ids, alpha, k)
    hit = torch.zeros(200, dtype=torch.bool)
    hit[[11, 90]] = True
    assert bool(out[hit].isnan().all()) and torch.equal(out[~hit], want[~hit])


def test_experts_refusals():
    d, E, inter, k_max = 128, 4, 64, 2
    w = experts_layer(4, d, E, inter)
    op = api.ExpertsFp8(w, d=d, E=E, inter=inter, k_max=k_max, max_tokens=8)
    h = normal(1, 8, d, dtype=BF16)
    ids, alpha, k = routing(1, 8, E, k_max)
    for args in ((normal(1, 9, d, dtype=BF16), *routing(1, 9, E, k_max)), (h.float(), ids, alpha, k),
                 (h, ids.long(), alpha, k), (h, ids, alpha[:, :1], k), (h, ids, alpha, k[:4])):
        with pytest.raises(ValueError):
            op.forward(*args)
    with pytest.raises(ValueError):
        api.ExpertsFp8(w, d=d, E=E, inter=inter, k_max=33, max_tokens=8)
    with pytest.raises(ValueError):
        api.ExpertsFp8(dict(w, w_down=w["w_down"][:3]), d=d, E=E, inter=inter, k_max=2,
                       max_tokens=8)
