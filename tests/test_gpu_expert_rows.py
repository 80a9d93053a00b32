"""Tokens to experts and back, and the gradients, against plain forms in 64 bits.

Tolerances, with u = 2^-24 and half = eps / 2 of the stored type: a sum of n products
in fp32, in any order, is off by (n + 1) u of the sum of magnitudes; a lane of a dot
product over d columns adds d / 32 + 8 terms and 5 shuffles.  Each output is rounded
once more, by half of its value.  Copies and whole numbers are exact."""
import numpy as np
import pytest
import torch

from paper_2608_01784_gb300 import _binding as B
from paper_2608_01784_gb300 import api

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF16, F32 = torch.bfloat16, torch.float32


def routing(seed, T, E, k_max, gaps=False, full=False):
    """ids with -1 in unused slots (anywhere, with gaps), weights that are NaN there."""
    rng = np.random.default_rng(seed)
    ids = rng.integers(0, E, (T, k_max)).astype(np.int32)
    used = (np.ones((T, k_max), bool) if full else rng.random((T, k_max)) < 0.6 if gaps else
            np.arange(k_max)[None] < rng.integers(0, k_max + 1, (T, 1)))
    ids[~used] = -1
    alpha = rng.random((T, k_max)).astype(np.float32)
    alpha[~used] = np.nan
    return torch.from_numpy(ids).cuda(), torch.from_numpy(alpha).cuda()


def plain_plan(ids, E):
    flat = ids.cpu().numpy().reshape(-1)
    key = np.where(flat >= 0, flat, E)
    order = np.argsort(key, kind="stable")
    n = int((flat >= 0).sum())
    row = np.full(flat.size, -1, np.int32)
    row[order[:n]] = np.arange(n)
    counts = np.bincount(key, minlength=E + 1)[:E]
    return row.reshape(ids.shape), counts, np.concatenate([[0], np.cumsum(counts)]), order[:n]


def draw(seed, dtype, *shape):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


def close(got, ref, bound, what):
    half = torch.finfo(got.dtype).eps / 2
    worst = ((got.double() - ref).abs() - half * ref.abs() - bound).max().item() if got.numel() else 0
    assert worst <= 0, (what, worst)


def pair_list(plan):
    """Tokens, slots and rows of the pairs."""
    t, j = torch.nonzero(plan.row_of >= 0, as_tuple=True)
    return t, j, plan.row_of[t, j].long()


def check_all(plan, alpha, d, dtype, seed=0):
    """Every call of a plan, on rows whose unused part is NaN."""
    T, cap = plan.T, plan.cap_rows
    t, j, r = pair_list(plan)
    x = draw(seed, dtype, T, d)
    to = torch.full((cap, d), 7.0, device="cuda", dtype=dtype)
    rows = api.expert_rows(x, plan, rows=to)
    want = torch.full((cap, d), 7.0, device="cuda", dtype=dtype)
    want[r] = x[t]
    assert rows is to and torch.equal(rows, want)

    y = torch.full((cap, d), float("nan"), device="cuda", dtype=dtype)
    y[r] = draw(seed + 1, dtype, cap, d)[r]
    n = plan.k_max + 2
    zero = torch.zeros((T, d), dtype=torch.float64, device="cuda")
    dx = api.expert_rows_backward(y, plan)
    close(dx, zero.index_add(0, t, y[r].double()),
          n * U * zero.index_add(0, t, y[r].double().abs()), "gradient of x")
    terms = y[r].double() * alpha[t, j].double()[:, None]
    out = api.expert_combine(y, alpha, plan)
    mag = zero.index_add(0, t, terms.abs())
    close(out, zero.index_add(0, t, terms), n * U * mag, "combine")
    res = draw(seed + 2, dtype, T, d)
    ref = zero.index_add(0, t, terms) + res.double()
    out = api.expert_combine(y, alpha, plan, residual=res)
    close(out, ref, n * U * (mag + res.double().abs()), "combine with residual")
    assert torch.equal(api.expert_combine(y, alpha, plan, residual=res, out=res), out)

    g = draw(seed + 3, dtype, T, d)
    to.fill_(7.0)
    d_rows, d_alpha = api.expert_combine_backward(g, y, alpha, plan, d_rows=to)
    want = torch.full((cap, d), 7.0, device="cuda", dtype=torch.float64)
    want[r] = g[t].double() * alpha[t, j].double()[:, None]
    close(d_rows, want, U * want.abs(), "gradient of the rows")
    left = torch.ones(cap, dtype=torch.bool, device="cuda")
    left[r] = False
    assert bool((d_rows[left] == 7).all())
    dots = torch.zeros(T, plan.k_max, dtype=torch.float64, device="cuda")
    size = torch.zeros_like(dots)
    dots[t, j] = (g[t].double() * y[r].double()).sum(1)
    size[t, j] = (g[t].double() * y[r].double()).abs().sum(1)
    close(d_alpha, dots, (d / 32 + 14) * U * size, "gradient of alpha")
    assert bool((d_alpha[plan.row_of < 0] == 0).all())
    again, _ = api.expert_combine_backward(g, y, alpha, plan, d_rows=y)
    assert again is y and torch.equal(again[r], d_rows[r])


@pytest.mark.parametrize("T,E,k_max,gaps", [
    (0, 8, 4, False), (1, 1, 1, False), (1, 64, 32, False), (5, 3, 7, True), (32, 64, 12, False),
    (85, 1024, 12, False), (86, 60, 12, False), (300, 8, 4, True), (999, 256, 12, True),
    (5000, 64, 12, False), (20000, 8, 8, True), (40001, 257, 12, False)])
def test_plans(T, E, k_max, gaps):
    ids, _ = routing(T + E, T, E, k_max, gaps)
    perm = torch.full((T * k_max,), -7, dtype=torch.int32, device="cuda")
    plan = api.expert_plan(ids, E=E, perm=perm)
    row, counts, offsets, order = plain_plan(ids, E)
    assert np.array_equal(plan.row_of.cpu().numpy(), row)
    assert np.array_equal(plan.counts.cpu().numpy(), counts)
    assert np.array_equal(plan.offsets.cpu().numpy(), offsets)
    got = perm.cpu().numpy()
    assert np.array_equal(got[:order.size], order) and (got[order.size:] == -7).all()
    assert plan.status() == B.REFLEX_OK
    # counts instead of marks: what lies behind them is not looked at
    if not gaps and T:
        k = (ids >= 0).sum(1).int()
        wild = torch.where(ids < 0, 1 << 30, ids)
        other = api.expert_plan(wild, E=E, k=k)
        assert torch.equal(other.row_of, plan.row_of) and other.status() == B.REFLEX_OK


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,d,E,k_max,gaps", [
    (1, 1, 1, 1, False), (3, 7, 2, 2, False), (40, 8, 64, 12, False), (33, 64, 8, 32, True),
    (257, 100, 60, 4, True), (100, 255, 8, 12, False), (64, 257, 64, 5, True),
    (31, 2048, 64, 12, False), (700, 1001, 256, 8, False), (12, 8192, 8, 12, True),
    (90, 1030, 16, 6, True)])
def test_shapes(T, d, E, k_max, gaps, dtype):
    ids, alpha = routing(T * 3 + d, T, E, k_max, gaps)
    check_all(api.expert_plan(ids, E=E), alpha, d, dtype)


@pytest.mark.parametrize("case", ["none used", "all used", "one expert", "same expert twice"])
def test_routings(case):
    ids, alpha = routing(1, 200, 16, 6, full=case != "none used")
    if case == "none used":
        ids.fill_(-1)
    if case == "one expert":
        ids.fill_(5)
    if case == "same expert twice":
        ids[:, 3] = ids[:, 1]
    check_all(api.expert_plan(ids, E=16), torch.nan_to_num(alpha, 0.5), 72, BF16)


def test_a_wrong_routing_is_reported():
    ids, _ = routing(2, 50, 8, 4, full=True)
    k = torch.full((50,), 4, dtype=torch.int32, device="cuda")
    assert api.expert_plan(ids, E=8, k=k).status() == B.REFLEX_OK
    wrong = ids.clone()
    wrong[7, 2] = 8
    for extra in (dict(), dict(k=k)):
        plan = api.expert_plan(wrong, E=8, **extra)
        assert plan.status() == B.REFLEX_EINVAL and int(plan.row_of[7, 2]) == -1
        assert int(plan.offsets[8]) == 199
    wrong[7, 2] = -1
    assert api.expert_plan(wrong, E=8).status() == B.REFLEX_OK
    plan = api.expert_plan(wrong, E=8, k=k)
    assert plan.status() == B.REFLEX_EINVAL and int(plan.offsets[8]) == 199
    for bad, pairs in ((5, 200), (-1, 196)):
        k[9] = bad
        plan = api.expert_plan(ids, E=8, k=k)
        assert plan.status() == B.REFLEX_EKRANGE and int(plan.offsets[8]) == pairs
    # the next plan clears the word
    k[9] = 4
    assert api.expert_plan(ids, E=8, k=k, plan=plan).status() == B.REFLEX_OK


def test_fewer_rows_than_pairs():
    ids, alpha = routing(3, 60, 8, 4, full=True)
    whole = api.expert_plan(ids, E=8)
    cut = api.expert_plan(ids, E=8, cap_rows=101)
    assert cut.status() == B.REFLEX_ECAPACITY
    want = torch.where(whole.row_of < 101, whole.row_of, -1)
    assert torch.equal(cut.row_of, want) and torch.equal(cut.offsets, whole.offsets)
    check_all(cut, alpha, 40, F32)
    none = api.expert_plan(ids, E=8, cap_rows=0)
    assert bool((none.row_of == -1).all())
    check_all(none, alpha, 40, F32)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d,ld,shift", [(64, 72, 0), (64, 71, 0), (64, 80, 1), (300, 304, 2)])
def test_strides_and_alignment(dtype, d, ld, shift):
    """The same bits as from packed rows; what lies between the rows stays as it is."""
    ids, alpha = routing(4, 90, 8, 6, gaps=True)
    plan = api.expert_plan(ids, E=8)
    x, y, g = draw(1, dtype, 90, d), draw(2, dtype, plan.cap_rows, d), draw(3, dtype, 90, d)

    def apart(t):
        wide = torch.full((t.shape[0], ld + shift), 7.0, device="cuda", dtype=dtype)
        wide[:, shift:shift + d] = t
        return wide, wide[:, shift:shift + d]
    wx, vx = apart(x)
    wy, vy = apart(y)
    wg, vg = apart(g)
    wr, vr = apart(torch.zeros_like(y))
    wo, vo = apart(torch.zeros_like(x))
    assert torch.equal(api.expert_rows(vx, plan, rows=vr),
                       api.expert_rows(x, plan, rows=torch.zeros_like(y)))
    assert torch.equal(api.expert_rows_backward(vy, plan, out=vo), api.expert_rows_backward(y, plan))
    assert torch.equal(api.expert_combine(vy, alpha, plan, residual=vx, out=vo),
                       api.expert_combine(y, alpha, plan, residual=x))
    vr.zero_()
    a = api.expert_combine_backward(vg, vy, alpha, plan, d_rows=vr)
    b = api.expert_combine_backward(g, y, alpha, plan, d_rows=torch.zeros_like(y))
    assert torch.equal(a[0], b[0])
    size = torch.zeros_like(alpha, dtype=torch.float64)
    t, j, r = pair_list(plan)
    size[t, j] = (g[t].double() * y[r].double()).abs().sum(1)
    # lanes share the columns in another order
    assert bool(((a[1] - b[1]).abs() <= 2 * (d / 32 + 14) * U * size).all())
    for wide, inner in ((wx, vx), (wy, vy), (wg, vg), (wr, vr), (wo, vo)):
        inner.fill_(7.0)
        assert bool((wide == 7.0).all())


def test_one_gradient_alone():
    """Either output of the gradient of the way back by itself (C entry point)."""
    ids, alpha = routing(8, 70, 8, 5)
    plan = api.expert_plan(ids, E=8)
    y, g = draw(1, BF16, plan.cap_rows, 96), draw(2, BF16, 70, 96)
    both = api.expert_combine_backward(g, y, alpha, plan, d_rows=torch.zeros_like(y))
    d_rows, d_alpha = torch.zeros_like(y), torch.full_like(alpha, 7.0)
    args = (B.REFLEX_DTYPE_BF16, g, 96, y, 96, alpha, plan.row_of, 70, 96, 5, plan.cap_rows)
    B.reflex_expert_combine_backward(*args, d_rows, 96, None)
    B.reflex_expert_combine_backward(*args, None, 0, d_alpha)
    assert torch.equal(d_rows, both[0]) and torch.equal(d_alpha, both[1])


def test_large_row_offsets():
    """Rows behind 2^31 elements."""
    T, d, k_max = 40000, 8192, 8
    ids = torch.randint(0, 64, (T, k_max), dtype=torch.int32, device="cuda")
    plan = api.expert_plan(ids, E=64)
    x = draw(1, BF16, T, d)
    rows = api.expert_rows(x, plan)
    assert rows.numel() > 1 << 31
    for t in (0, 1, T // 2, T - 1):
        for j in (0, k_max - 1):
            assert torch.equal(rows[plan.row_of[t, j].long()], x[t])
    back = api.expert_rows_backward(rows, plan)
    close(back, 8 * x.double(), 0.0, "eight times x")
    alpha = torch.full((T, k_max), 0.125, device="cuda")
    d_rows, d_alpha = api.expert_combine_backward(x, rows, alpha, plan, d_rows=rows)
    last = plan.row_of[:, k_max - 1].long()
    assert torch.equal(d_rows[last], x * 0.125)


def test_differences():
    """alpha's and the rows' gradients: the sum is linear in each, so a difference of
    the formula in 64 bits along a direction is the slope itself."""
    ids, alpha = routing(5, 30, 8, 5)
    plan = api.expert_plan(ids, E=8)
    t, j, r = pair_list(plan)
    y, g = draw(1, F32, plan.cap_rows, 48), draw(2, F32, 30, 48)
    d_rows, d_alpha = api.expert_combine_backward(g, y, alpha, plan)
    v, w = draw(3, F32, plan.cap_rows, 48).double(), draw(4, F32, 30, 5).double()

    def total(rows, a):
        return (rows[r] * a[t, j][:, None] * g[t].double()).sum().item()
    yd, ad = y.double(), alpha.double()
    for got, slope in (((d_rows[r].double() * v[r]), total(yd + v, ad) - total(yd, ad)),
                       ((d_alpha[t, j].double() * w[t, j]), total(yd, ad + w) - total(yd, ad))):
        assert abs(got.sum().item() - slope) <= 16 * U * got.abs().sum().item() + 1e-9


def test_streams_and_graphs():
    ids, alpha = routing(6, 3000, 64, 8, full=True)
    x, g = draw(1, BF16, 3000, 128), draw(2, BF16, 3000, 128)

    def run(stream=None):
        plan = api.expert_plan(ids, E=64, stream=stream)
        rows = api.expert_rows(x, plan, stream=stream)
        out = api.expert_combine(rows, alpha, plan, residual=x, stream=stream)
        dr, da = api.expert_combine_backward(g, rows, alpha, plan, stream=stream)
        dx = api.expert_rows_backward(dr, plan, stream=stream)
        return plan.row_of, rows, out, dr, da, dx
    want = run()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = run(s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    # two graphs, each with its own workspaces, replayed side by side
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            graphs.append((graph, run()))
    for _, outs in graphs:
        for t in outs:
            t.zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in graphs]
    for (graph, _), s in zip(graphs, streams):
        with torch.cuda.stream(s):
            graph.replay()
    torch.cuda.synchronize()
    for _, outs in graphs:
        assert all(torch.equal(a, b) for a, b in zip(want, outs))


def test_refusals(monkeypatch):
    ids, alpha = routing(7, 6, 4, 3, full=True)
    plan = api.expert_plan(ids, E=4)
    x, rows = draw(1, F32, 6, 10), draw(2, F32, 18, 10)

    def enqueued(*args, **kw):
        raise AssertionError("the call went on")
    for name in ("reflex_expert_plan", "reflex_expert_rows", "reflex_expert_combine",
                 "reflex_expert_combine_backward"):
        monkeypatch.setattr(B, name, enqueued)
    calls = [
        lambda: api.expert_plan(ids.long(), E=4), lambda: api.expert_plan(ids.T, E=4),
        lambda: api.expert_plan(ids.cpu(), E=4), lambda: api.expert_plan(ids, E=1025),
        lambda: api.expert_plan(ids, E=8, plan=plan),
        lambda: api.expert_plan(ids, E=4, k=torch.ones(5, dtype=torch.int32, device="cuda")),
        lambda: api.expert_plan(ids, E=4, perm=torch.ones(17, dtype=torch.int32, device="cuda")),
        lambda: api.expert_rows(x[:5], plan), lambda: api.expert_rows(x, plan, rows=rows[:17]),
        lambda: api.expert_rows(x, plan, rows=rows[:, :9]),
        lambda: api.expert_rows(x, plan, rows=rows.bfloat16()), lambda: api.expert_rows(x.T, plan),
        lambda: api.expert_rows_backward(rows[:17], plan),
        lambda: api.expert_combine(rows, alpha.double(), plan),
        lambda: api.expert_combine(rows, alpha[:5], plan),
        lambda: api.expert_combine(rows, alpha, plan, residual=x[:, :9]),
        lambda: api.expert_combine(rows, alpha, plan, out=x.bfloat16()),
        lambda: api.expert_combine_backward(x[:5], rows, alpha, plan),
        lambda: api.expert_combine_backward(x, rows, alpha, plan, d_rows=rows[:, :9]),
        lambda: api.expert_combine_backward(x, rows, alpha, plan, d_alpha=alpha.double())]
    for i, c in enumerate(calls):
        with pytest.raises(ValueError):
            c()
            pytest.fail(f"call {i} went on")
