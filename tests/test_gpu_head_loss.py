"""The loss of a vocabulary head and its gradients against the formulas in 64 bits.

Inputs are small whole numbers times a power of two and not negative, so that every
logit is exact in fp32 and no tile's part of a gradient hides in cancellation.
Tolerances, with u = 2^-24: a sum of exponentials over the vocabulary adds at most 8 + 3
+ 4 terms in a slice of 128 columns, then a slice in 32, then 32; an exponential is off by
4 u and the rounding of its exponent (2 u times its size); so lse and loss are off by
SUM = (64 + vocab / 2048) u and a few u of lse.  G is off by half a step of bf16 (2^-8)
and by p times DELTA = (8 + 4 (|z| + |lse|)) u; n products add n u of the sum of their
magnitudes (2 n u for the tensor cores, which cut instead of rounding); an output is
rounded once more, by half of its value."""
import math

import pytest
import torch

from paper_2608_01784_gb300 import _binding as B
from paper_2608_01784_gb300 import api

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF16, F32 = torch.bfloat16, torch.float32


def make(seed, rows, vocab, k, masked=1.0, ld=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    scale = 2.0 ** -round(math.log2(4.5 * math.sqrt(k) / 2))
    ld = -(-k // 8) * 8 if ld is None else ld
    w = torch.full((vocab, ld), float("nan"), device="cuda", dtype=BF16)
    w[:, :k] = torch.randint(0, 5, (vocab, k), generator=g, device="cuda") * scale
    h = torch.randint(0, 5, (rows, k), generator=g, device="cuda").to(BF16)
    t = torch.randint(0, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
    live = torch.rand(rows, generator=g, device="cuda") < masked
    t = torch.where(live, t, -1 - t)
    h[~live] = float("nan")  # not read
    grad = torch.where(live, torch.rand(rows, generator=g, device="cuda") + 0.5, float("nan"))
    return h, w[:, :k], t, grad


def formula(h, w, t):
    """Of the rows with a target: (their numbers, z, lse) in 64 bits."""
    i = torch.nonzero(t >= 0)[:, 0]
    z = h[i].double() @ w.double().T
    return i, z, torch.logsumexp(z, 1)


def check_loss(h, w, t, loss, lse):
    i, z, ref = formula(h, w, t)
    tol = (64 + w.shape[0] / 2048) * U + 4 * U * ref.abs()
    want = ref - z.gather(1, t[i].long()[:, None])[:, 0]
    assert bool(((lse[i].double() - ref).abs() <= tol).all())
    # the loss is larger than lse where the target is far below: its own two roundings, of
    # the difference and of the sum, are u |loss| each (fp32 has no value nearer to 3014.5497
    # than 9e-5, where 4 u lse is 2e-6)
    tol = tol + 2 * U * want.abs()
    assert bool(((loss[i].double() - want).abs() <= tol).all()), (loss[i] - want).abs().max()
    rest = torch.ones_like(t, dtype=torch.bool)
    rest[i] = False
    assert not loss[rest].any() and not lse[rest].any()


def check_grad(h, w, t, grad, dh, dw):
    i, z, lse = formula(h, w, t)
    p, c, hd, wd = torch.exp(z - lse[:, None]), grad[i].double()[:, None], h[i].double(), w.double()
    delta = (8 + 4 * (z.abs() + lse[:, None].abs())) * U
    off = c * p * delta
    p[torch.arange(i.numel()), t[i].long()] -= 1
    G = c * p
    size = G.abs()
    for got, ref, mag, n in ((dh, G @ wd, lambda e: e @ wd.abs(), w.shape[0]),
                             (dw, G.T @ hd, lambda e: e.T @ hd.abs(), i.numel())):
        if got is None:
            continue
        rows = got if got is dw else got[i]
        half = torch.finfo(got.dtype).eps / 2
        bound = mag(size * (2.0 ** -8 + 2 * n * U) + off) + half * ref.abs()
        worst = ((rows.double() - ref).abs() - bound).max().item() if ref.numel() else 0
        assert worst <= 0, ("dw" if got is dw else "dh", worst)
    if dh is not None:
        rest = torch.ones_like(t, dtype=torch.bool)
        rest[i] = False
        assert not dh[rest].any()


def run(h, w, t, grad, **kw):
    loss, lse = api.head_loss(h, w, t)
    return loss, lse, *api.head_loss_backward(h, w, t, lse, grad, **kw)


SHAPES = [(1, 1, 1), (1, 2, 1), (2, 5, 8), (3, 300, 17), (32, 1000, 64), (33, 257, 65),
          (128, 256, 128), (129, 511, 256), (255, 1025, 250), (256, 2048, 512), (257, 4099, 130),
          (600, 3001, 320), (1000, 700, 2048), (5, 20000, 96), (2000, 1, 40), (31, 1500, 5000),
          (64, 20000, 130), (65, 20000, 130), (50, 70001, 96), (1, 128, 1100), (17, 385, 700)]


@pytest.mark.parametrize("rows,vocab,k", SHAPES)
def test_loss(rows, vocab, k):
    for masked in (1.0, 0.5):
        h, w, t, _ = make(rows + vocab, rows, vocab, k, masked)
        status = torch.full((1,), 77, dtype=torch.int32, device="cuda")
        check_loss(h, w, t, *api.head_loss(h, w, t, status=status))
        assert B.reflex_read_status(status) == B.REFLEX_OK


@pytest.mark.parametrize("rows,vocab,k", SHAPES)
def test_gradient(rows, vocab, k):
    for masked in (1.0, 0.5):
        h, w, t, grad = make(rows + vocab, rows, vocab, k, masked)
        _, lse = api.head_loss(h, w, t)
        status = torch.full((1,), 77, dtype=torch.int32, device="cuda")
        dh, dw = api.head_loss_backward(h, w, t, lse, grad, status=status)
        assert B.reflex_read_status(status) == B.REFLEX_OK
        check_grad(h, w, t, grad, dh, dw)


@pytest.mark.parametrize("rows,vocab,k", [(8192, 9001, 136), (4100, 35000, 72), (20000, 5000, 64),
                                          (3, 263000, 16), (8192, 33000, 40),
                                          (20000, 14000, 64), (3, 1050000, 16)])
def test_several_pieces(rows, vocab, k):
    h, w, t, grad = make(rows, rows, vocab, k, 0.9)
    loss, lse, dh, dw = run(h, w, t, grad)
    check_loss(h, w, t, loss, lse)
    check_grad(h, w, t, grad, dh, dw)


@pytest.mark.parametrize("dtype_h,dtype_w", [(F32, F32), (F32, BF16), (BF16, F32)])
@pytest.mark.parametrize("rows,vocab,k", [(40, 700, 100), (300, 300, 33)])
def test_gradients_in_fp32(rows, vocab, k, dtype_h, dtype_w):
    h, w, t, grad = make(1, rows, vocab, k, 0.7)
    dh = torch.full((rows, k), 7.0, device="cuda", dtype=dtype_h)
    dw = torch.full((vocab, k), 7.0, device="cuda", dtype=dtype_w)
    got = run(h, w, t, grad, d_hidden=dh, d_weight=dw)[2:]
    assert got[0] is dh and got[1] is dw
    check_grad(h, w, t, grad, dh, dw)


@pytest.mark.parametrize("need", [(True, False), (False, True)])
@pytest.mark.parametrize("rows,vocab,k", [(70, 900, 120), (8192, 9001, 64)])
def test_one_gradient(rows, vocab, k, need):
    h, w, t, grad = make(2, rows, vocab, k, 0.8)
    both = run(h, w, t, grad)[2:]
    one = run(h, w, t, grad, need_hidden=need[0], need_weight=need[1])[2:]
    for a, b, n in zip(both, one, need):
        assert torch.equal(a, b) if n else b is None


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("k,ldh,ldw,ldd", [(64, 64, 72, 64), (64, 67, 64, 65), (100, 101, 104, 103),
                                           (129, 200, 136, 131), (60, 64, 64, 64)])
def test_strides(k, ldh, ldw, ldd, dtype):
    """What lies between rows is neither used nor written; d_weight of any stride."""
    rows, vocab = 150, 777
    h, w, t, grad = make(3, rows, vocab, k, 0.8, ld=ldw)
    wide = torch.full((rows, ldh), float("nan"), device="cuda", dtype=BF16)
    wide[:, :k] = h
    dh = torch.full((rows, ldd), 7.0, device="cuda", dtype=dtype)
    dw = torch.full((vocab, ldd), 7.0, device="cuda", dtype=dtype)
    loss, lse, _, _ = run(wide[:, :k], w, t, grad, d_hidden=dh[:, :k], d_weight=dw[:, :k])
    check_loss(h, w, t, loss, lse)
    check_grad(h, w, t, grad, dh[:, :k], dw[:, :k])
    assert bool((dh[:, k:] == 7).all()) and bool((dw[:, k:] == 7).all())


def test_gradients_at_odd_addresses():
    h, w, t, grad = make(4, 90, 500, 72)
    want = run(h, w, t, grad)[2:]
    dh, dw = (torch.full((n * 72 + 1,), 7.0, device="cuda", dtype=BF16) for n in (90, 500))
    run(h, w, t, grad, d_hidden=dh[1:].view(90, 72), d_weight=dw[1:].view(500, 72))
    assert torch.equal(dh[1:].view(90, 72), want[0]) and torch.equal(dw[1:].view(500, 72), want[1])
    assert float(dh[0]) == float(dw[0]) == 7.0


@pytest.mark.parametrize("rows", [1, 40, 300])
def test_no_row_counts(rows):
    h, w, t, grad = make(5, rows, 600, 64)
    t.fill_(-1)
    loss, lse, dh, dw = run(h, w, t, grad)
    for x in (loss, lse, dh, dw):
        assert not x.any()


@pytest.mark.parametrize("rows", [40, 300])
def test_the_rows_gradient_in_place(rows):
    h, w, t, grad = make(13, rows, 500, 64, 0.8)
    want = run(h, w, t, grad)[2:]
    got = run(h, w, t, grad, d_hidden=h)[2:]
    assert got[0] is h and torch.equal(h, want[0]) and torch.equal(got[1], want[1])


def test_no_rows():
    h, w, t, grad = make(6, 0, 600, 60)
    loss, lse, dh, dw = run(h, w, t, grad)
    assert loss.shape == lse.shape == (0,) and dh.shape == (0, 60)
    assert dw.shape == (600, 60) and not dw.any()


def test_targets_outside_the_vocabulary():
    h, w, t, grad = make(7, 100, 300, 64)
    t[13], t[77] = 300, 1 << 30
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    loss, lse = api.head_loss(h, w, t, status=status)
    assert B.reflex_read_status(status) == B.REFLEX_EINVAL
    dh, dw = api.head_loss_backward(h, w, t, lse, grad, status=status)
    assert B.reflex_read_status(status) == B.REFLEX_EINVAL
    t[13] = t[77] = -1
    check_loss(h, w, t, loss, lse)
    check_grad(h, w, t, grad, dh, dw)
    api.head_loss(h, w, t, status=status)
    assert B.reflex_read_status(status) == B.REFLEX_OK


def test_the_same_bits():
    """On every run, and for a row whatever the others are."""
    h, w, t, grad = make(8, 3000, 5000, 128, 0.7)
    a, b = run(h, w, t, grad), run(h, w, t, grad)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    few = slice(1111, 1300)
    loss, lse = api.head_loss(h[few], w, t[few].contiguous())
    assert torch.equal(loss, a[0][few]) and torch.equal(lse, a[1][few])
    # up to 64 rows in an order of their own
    few = slice(1111, 1170)
    a, b = (run(h[few], w, t[few].contiguous(), grad[few].contiguous()) for _ in range(2))
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    loss, lse = api.head_loss(h[1120:1163], w, t[1120:1163].contiguous())
    assert torch.equal(loss, a[0][9:52]) and torch.equal(lse, a[1][9:52])


@pytest.mark.parametrize("rows", [40, 500])
def test_a_row_that_is_not_finite_stays_by_itself(rows):
    h, w, t, grad = make(9, rows, 900, 64)
    loss, lse = api.head_loss(h, w, t)
    h[17, 3], h[30, 5] = float("nan"), float("inf")
    a, b = api.head_loss(h, w, t)
    keep = torch.ones(rows, dtype=torch.bool, device="cuda")
    keep[17] = keep[30] = False
    assert torch.equal(a[keep], loss[keep]) and torch.equal(b[keep], lse[keep])
    assert not a[~keep].isfinite().any()


@pytest.mark.parametrize("far", [60.0, 3000.0, 1e6])
def test_logits_far_apart(far):
    """Rows that are sure of a token: its loss is 0, another's the distance."""
    vocab, k = 700, 64
    h = torch.zeros(4, k, device="cuda", dtype=BF16)
    h[:, 0] = far
    w = torch.zeros(vocab, k, device="cuda", dtype=BF16)
    w[500, 0] = 1.0
    far = float(h[0, 0])
    t = torch.tensor([500, 0, 699, 500], dtype=torch.int32, device="cuda")
    for sign in (1.0, -1.0):
        check_loss(h * sign, w, t, *api.head_loss(h * sign, w, t))
    loss, lse = api.head_loss(h, w, t)
    assert loss.tolist()[0] <= 1e-6 and abs(loss.tolist()[1] - far) <= 4 * U * far
    grad = torch.ones(4, device="cuda")
    check_grad(h, w, t, grad, *api.head_loss_backward(h, w, t, lse, grad))


def test_random_values():
    """Values as a model has them: relative errors over whole outputs.  G's rounding and
    the output's are each below 2^-8; the logits' sums in fp32 are far below that."""
    g = torch.Generator(device="cuda").manual_seed(1)
    h = torch.randn(700, 512, generator=g, device="cuda").to(BF16)
    w = (torch.randn(6001, 512, generator=g, device="cuda") * 0.08).to(BF16)
    t = torch.randint(0, 6001, (700,), generator=g, device="cuda", dtype=torch.int32)
    grad = torch.rand(700, generator=g, device="cuda") / 700
    loss, lse, dh, dw = run(h, w, t, grad)
    i, z, ref = formula(h, w, t)
    want = ref - z.gather(1, t.long()[:, None])[:, 0]
    assert float((loss.double() - want).norm() / want.norm()) <= 1e-6
    p = torch.exp(z - ref[:, None])
    p[i, t.long()] -= 1
    G = grad.double()[:, None] * p
    for got, r in ((dh, G @ w.double()), (dw, G.T @ h.double())):
        assert float((got.double() - r).norm() / r.norm()) <= 2.0 ** -7


def test_differences():
    """Gradients against central differences of the formula in 64 bits along a direction;
    2^-7 of the terms for the two roundings to bf16, 1e-6 for the difference."""
    h, w, t, grad = make(10, 40, 300, 64, 0.8)
    _, _, dh, dw = run(h, w, t, grad)
    i = torch.nonzero(t >= 0)[:, 0]
    g = torch.Generator(device="cuda").manual_seed(2)

    def total(a, b):
        z = a @ b.T
        return ((torch.logsumexp(z, 1) - z.gather(1, t[i].long()[:, None])[:, 0])
                * grad[i].double()).sum().item()
    hd, wd = h[i].double(), w.double()
    for got, at in ((dh[i], hd), (dw, wd)):
        v = torch.randn(at.shape, generator=g, device="cuda", dtype=torch.float64)
        ends = [total(hd + s * v, wd) if at is hd else total(hd, wd + s * v) for s in (1e-4, -1e-4)]
        slope = (ends[0] - ends[1]) / 2e-4
        terms = (got.double() * v)
        assert abs(terms.sum().item() - slope) <= 2.0 ** -7 * terms.abs().sum().item() + 1e-6


@pytest.mark.parametrize("rows", [60, 500])
def test_streams_and_graphs(rows):
    h, w, t, grad = make(11, rows, 3000, 256, 0.6)
    want = run(h, w, t, grad)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    loss, lse = api.head_loss(h, w, t, stream=s)
    dh, dw = api.head_loss_backward(h, w, t, lse, grad, stream=s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (loss, lse, dh, dw)))
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            graphs.append((graph, run(h, w, t, grad)))
    for _, outs in graphs:
        for x in outs:
            x.fill_(7.0)
    torch.cuda.synchronize()
    for (graph, _), s in zip(graphs, [torch.cuda.Stream(), torch.cuda.Stream()]):
        with torch.cuda.stream(s):
            graph.replay()
    torch.cuda.synchronize()
    for _, outs in graphs:
        assert all(torch.equal(a, b) for a, b in zip(want, outs))


def test_refusals(monkeypatch):
    h, w, t, grad = make(12, 6, 30, 16)
    lse = torch.zeros(6, device="cuda")

    def enqueued(*args, **kw):
        raise AssertionError("the call went on")
    monkeypatch.setattr(B, "reflex_head_loss", enqueued)
    monkeypatch.setattr(B, "reflex_head_loss_backward", enqueued)
    odd = torch.zeros(30, 17, device="cuda", dtype=BF16)[:, :16]
    shifted = torch.zeros(30 * 16 + 1, device="cuda", dtype=BF16)[1:].view(30, 16)
    calls = [lambda: api.head_loss(h.float(), w, t), lambda: api.head_loss(h, w.float(), t),
             lambda: api.head_loss(h, w[:, :8], t), lambda: api.head_loss(h, odd, t),
             lambda: api.head_loss(h, shifted, t), lambda: api.head_loss(h, w, t.long()),
             lambda: api.head_loss(h, w, t[:5]), lambda: api.head_loss(h, w, t.cpu()),
             lambda: api.head_loss(h.T, w, t), lambda: api.head_loss(h, w[:0], t),
             lambda: api.head_loss(h, w, t, loss=lse[:5]),
             lambda: api.head_loss(h, w, t, lse=lse.double()),
             lambda: api.head_loss(h, w, t, status=torch.zeros(2, dtype=torch.int32, device="cuda")),
             lambda: api.head_loss_backward(h, w, t, lse[:5], grad),
             lambda: api.head_loss_backward(h, w, t, lse, grad.double()),
             lambda: api.head_loss_backward(h, w, t, lse, grad, d_hidden=h[:5]),
             lambda: api.head_loss_backward(h, w, t, lse, grad, d_weight=w.half()),
             lambda: api.head_loss_backward(h, w, t, lse, grad, d_weight=w),
             lambda: api.head_loss_backward(h, w, t, lse, grad, need_hidden=False,
                                            need_weight=False),
             lambda: api.head_loss_backward(h, w, t, lse, grad, need_weight=False,
                                            d_weight=w.clone())]
    for i, c in enumerate(calls):
        with pytest.raises(ValueError):
            c()
            pytest.fail(f"call {i} went on")
