"""Sampling on the GPU against its definition written out with numpy: the
weights by separate fp32 operations, every decision on 64-bit integers, the
token equal; the confidence against the softmax in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2608_01784_gb300 import _binding as B
from paper_2608_01784_gb300 import api

pytestmark = pytest.mark.gpu

F = np.float32
BF16, F32 = torch.bfloat16, torch.float32
COEF = [F(c) for c in (0.6931471824645996, 0.2402234971523285, 0.055503811687231064,
                       0.00966636836528778, 0.0013381302123889327)]


def weights(z, m, T):
    with np.errstate(all="ignore"):
        c = min(F(1.442695021629333) / F(T), np.finfo(F).max)
        t = (z - m).astype(F) * c
        t = np.where(t > -40, t, F(-40)).astype(F)
        n = np.rint(t)
        f = (t - n).astype(F)
        p = np.full_like(f, COEF[4])
        for c_i in (COEF[3], COEF[2], COEF[1], COEF[0], F(1)):
            p = (p * f).astype(F) + c_i
        return np.floor(np.ldexp(p.astype(np.float64), n.astype(int) + 31)).astype(np.int64)


def reference(z, T, k, p, min_p, u):
    """(token, confidence) of one row of fp32 logits."""
    z = np.where(np.isnan(z), F(-np.inf), z).astype(F)
    m = z.max()
    if m == -np.inf:
        return -1, 0.0
    if m == np.inf:
        z, m = np.where(z == np.inf, F(0), F(-np.inf)).astype(F), F(0)
    e = np.exp(z.astype(np.float64) - np.float64(m))
    if T == 0:
        tok = int(np.argmax(z))
        return tok, e[tok] / e.sum()
    w = weights(z, m, T)
    order = np.argsort(-z, kind="stable")
    q = w[order]
    keep = np.ones(z.size, bool)
    if k > 0:
        keep &= np.arange(z.size) < k
    if p < 1:
        qk = np.where(keep, q, 0)
        before = np.cumsum(qk) - qk
        keep &= before.astype(np.float64) < np.float64(F(p)) * np.float64(qk.sum())
    if min_p > 0:
        keep &= q >= np.ceil(np.float64(F(min_p)) * 2.0 ** 31)
    kept = np.zeros_like(w)
    kept[order] = np.where(keep, q, 0)
    run = np.cumsum(kept).astype(np.float64)
    u = min(max(F(u), F(0)), F(1) - F(2.0 ** -24))
    tok = int(np.argmax(run > np.float64(u) * run[-1]))
    return tok, e[tok] / e.sum()


def check(logits, u, T=None, k=None, p=None, min_p=None, masked=None):
    rows = logits.shape[0]
    dev = lambda x, dt: None if x is None else torch.tensor(x, dtype=dt, device="cuda")  # noqa: E731
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    tokens, conf = api.sample(logits, dev(u, F32), temperature=dev(T, F32),
                              top_k=dev(k, torch.int32), top_p=dev(p, F32), min_p=dev(min_p, F32),
                              masked=dev(masked, torch.uint8), status=status)
    assert B.reflex_read_status(status) == B.REFLEX_OK
    z = logits.float().cpu().numpy()
    tokens, conf = tokens.cpu().numpy(), conf.cpu().numpy()
    pick = lambda x, r, other: other if x is None else x[r]  # noqa: E731
    for r in range(rows):
        if masked is not None and not masked[r]:
            assert tokens[r] == -1 and conf[r] == 0
            continue
        tok, c = reference(z[r], F(pick(T, r, 1)), pick(k, r, 0), pick(p, r, 1), pick(min_p, r, 0),
                           u[r])
        assert tokens[r] == tok, (r, tokens[r], tok)
        # the chosen logit's distance from the largest, in fp32, times its exponent's
        # relative step, and fp32 sums of up to 200 terms a thread
        far = 0.0 if tok < 0 or not np.isfinite(z[r][tok]) else float(np.nanmax(z[r]) - z[r][tok])
        tol = c * (200 * 2.0 ** -24 + (2 + far) * 2.0 ** -22) + 2e-38
        assert abs(float(conf[r]) - c) <= tol, (r, conf[r], c)


def logits_of(seed, rows, vocab, dtype=F32, std=2.0, peak=8.0):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn(rows, vocab, generator=g) * std
    at = torch.randint(0, vocab, (rows, min(vocab, 12)), generator=g)
    z.scatter_(1, at, torch.rand(at.shape, generator=g) * peak)
    return z.to(dtype).cuda()


def uniforms(seed, n):
    return np.random.default_rng(seed).random(n).astype(F)


VOCABS = [1, 2, 7, 8, 9, 255, 256, 1000, 2041, 2048, 2049, 4097, 50001, 131072, 262144]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab", VOCABS)
def test_vocabularies(vocab, dtype):
    rows = 12
    z = logits_of(vocab, rows, vocab, dtype)
    u = uniforms(vocab, rows)
    g = np.random.default_rng(vocab)
    check(z, u)
    check(z, u, T=g.choice([0.0, 0.3, 0.7, 1.0, 1.5], rows), k=g.choice([0, 1, 5, 50, 999], rows),
          p=g.choice([0.1, 0.5, 0.9, 0.99, 1.0], rows), min_p=g.choice([0.0, 0.01, 0.2], rows))


@pytest.mark.parametrize("rows", [1, 3, 40, 300])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("filters", ["k", "p", "m", "kp", "kpm"])
def test_filters(rows, dtype, filters):
    vocab = 3001
    z = logits_of(rows, rows, vocab, dtype, std=1.0, peak=5.0)
    g = np.random.default_rng(rows + len(filters))
    check(z, uniforms(rows, rows), T=g.uniform(0.3, 2.0, rows).astype(F),
          k=g.integers(1, 400, rows) if "k" in filters else None,
          p=g.uniform(0.05, 1.0, rows).astype(F) if "p" in filters else None,
          min_p=g.uniform(0.0, 0.5, rows).astype(F) if "m" in filters else None)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("levels", [1, 2, 5, 40])
def test_ties_go_by_index(levels, dtype):
    """Few distinct logits: the last kept token lies among equal ones."""
    rows, vocab = 64, 5000
    g = torch.Generator().manual_seed(levels)
    z = (torch.randint(0, levels, (rows, vocab), generator=g).float() * 0.25).to(dtype).cuda()
    r = np.random.default_rng(levels)
    check(z, uniforms(1, rows), k=r.integers(1, 5000, rows))
    check(z, uniforms(2, rows), p=r.uniform(0.01, 1.0, rows).astype(F))
    check(z, uniforms(3, rows), T=r.uniform(0.1, 3, rows).astype(F), k=r.integers(1, 5000, rows),
          p=r.uniform(0.01, 1.0, rows).astype(F), min_p=r.uniform(0, 1, rows).astype(F))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_wide_and_flat_rows(dtype):
    """Cuts that fall far down a flat row, logits of any size, exact powers, both zeros."""
    g = torch.Generator().manual_seed(5)
    vocab = 9000
    rows = [torch.randn(vocab, generator=g) * s for s in (1e-6, 1e-3, 0.05, 10, 1e4, 1e30)]
    rows += [torch.linspace(-1, 1, vocab), torch.linspace(-30, 0, vocab),
             torch.where(torch.arange(vocab) % 3 == 0, -0.0, 0.0),
             torch.cat([torch.zeros(1), torch.full((vocab - 1,), -25.0)]),
             torch.randn(vocab, generator=g) * 1e-40, 100 + torch.randn(vocab, generator=g)]
    z = torch.stack(rows).to(dtype).cuda()
    n = z.shape[0]
    for k in (1, 17, 4500, 8999, 9000, 20000):
        check(z, uniforms(k, n), k=np.full(n, k))
    for p in (1e-30, 0.1, 0.5, 0.999, 1.0, 2.0):
        check(z, uniforms(3, n), p=np.full(n, p, F))
        check(z, uniforms(4, n), p=np.full(n, p, F), k=np.full(n, 6000), T=np.full(n, 3.0, F))
    for T in (0.0, 1e-38, 1e-6, 0.01, 50.0, 1e30):
        check(z, uniforms(5, n), T=np.full(n, T, F), p=np.full(n, 0.7, F))
    for m in (-1.0, 1e-9, 0.999, 1.0):
        check(z, uniforms(6, n), min_p=np.full(n, m, F))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab", [10, 3000])
def test_masked_logits(dtype, vocab):
    g = torch.Generator().manual_seed(vocab)
    z = torch.randn(10, vocab, generator=g)
    inf = float("inf")
    z[0] = -inf                       # nothing left
    z[1] = float("nan")
    z[2, 1:] = -inf                   # one token left
    z[3, ::2] = float("nan")
    z[4, 3] = inf                     # those alone
    z[4, 7] = inf
    z[5] = torch.finfo(dtype).min     # masked by the lowest value, all of it
    z[6, : vocab - 2] = torch.finfo(dtype).min
    z[7, 5] = inf
    z[7, 6] = float("nan")
    z[8, : vocab // 2] = -inf
    z[9] = inf
    z = z.to(dtype).cuda()
    for kw in ({}, dict(k=np.full(10, 3)), dict(p=np.full(10, 0.6, F)),
               dict(T=np.zeros(10, F)), dict(min_p=np.full(10, 0.4, F)),
               dict(k=np.full(10, 2), p=np.full(10, 0.9, F), T=np.full(10, 0.5, F))):
        check(z, uniforms(len(kw), 10), **kw)


def test_uniforms_at_their_ends():
    z = logits_of(3, 6, 700)
    u = np.array([0.0, 1.0 - 2.0 ** -24, 1.0, 5.0, -1.0, 0.5], F)
    check(z, u)
    check(z, u, p=np.full(6, 0.8, F))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab,offset,extra", [(1001, 1, 0), (1000, 3, 5), (4096, 1, 1), (77, 7, 9)])
def test_strides_and_alignment(dtype, vocab, offset, extra):
    rows = 9
    z = logits_of(vocab, rows, vocab, dtype)
    flat = torch.full((rows * (vocab + extra) + offset + 8,), 1e9, dtype=dtype, device="cuda")
    view = flat[offset:offset + rows * (vocab + extra)].view(rows, vocab + extra)[:, :vocab]
    view.copy_(z)
    u = uniforms(vocab, rows)
    check(view, u, p=np.full(rows, 0.9, F))
    check(view, u, masked=(np.arange(rows) % 2).astype(np.uint8))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_row_is_the_same_in_any_batch(dtype):
    """Few rows are split over more CTAs than many."""
    z = logits_of(11, 700, 20011, dtype)
    u = torch.tensor(uniforms(1, 700), device="cuda")
    T = torch.full((700,), 0.9, device="cuda")
    p = torch.full((700,), 0.97, device="cuda")
    many, _ = api.sample(z, u, temperature=T, top_p=p)
    for r in (0, 1, 350, 699):
        one, _ = api.sample(z[r:r + 1], u[r:r + 1], temperature=T[r:r + 1], top_p=p[r:r + 1])
        assert int(one[0]) == int(many[r])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab,extra", [(60000, 8), (60001, 0), (33333, 3)])
def test_many_long_rows(dtype, vocab, extra):
    """Enough rows that a CTA walks each in global memory: every kind of row and filter."""
    rows = 90
    flat = torch.full((rows, vocab + extra), 1e9, dtype=dtype, device="cuda")
    z = flat[:, :vocab]
    z.copy_(logits_of(vocab, rows, vocab, dtype))
    inf = float("inf")
    z[3] = -inf
    z[4] = float("nan")
    z[5, ::3] = float("nan")
    z[6, vocab - 1] = inf
    z[6, 9] = inf
    z[6, 10] = float("nan")
    z[7] = 0.25
    z[8] = torch.finfo(dtype).min
    z[9, : vocab - 5] = -inf
    z[10] = (torch.arange(vocab, device="cuda") % 7).to(dtype)
    z[11] = (torch.linspace(0, 20, vocab, device="cuda")).to(dtype)
    z[12, 100] = 60.0
    g = np.random.default_rng(vocab)
    u = uniforms(vocab, rows)
    masked = (g.random(rows) < 0.7).astype(np.uint8)
    T = g.choice([0.0, 0.5, 1.0, 1.4], rows).astype(F)
    k = g.choice([0, 1, 60, 2500, 20000, 59999], rows)
    p = g.choice([0.2, 0.9, 0.97, 0.9999, 1.0], rows).astype(F)
    min_p = g.choice([0.0, 0.0, 0.03, 0.5], rows).astype(F)
    check(z, u)
    check(z, u, T=T, masked=masked)
    check(z, u, k=k)
    check(z, u, p=p, T=T)
    check(z, u, min_p=min_p, p=p)
    check(z, u, T=T, k=k, p=p, min_p=min_p)


@pytest.mark.parametrize("T,p", [(1.0, 1.0), (0.7, 1.0), (1.3, 0.8)])
def test_frequencies(T, p):
    """Evenly spaced uniforms give each token its share to within one draw."""
    n, vocab = 4096, 60
    z = logits_of(2, 1, vocab, F32, std=1.0, peak=2.0).expand(n, vocab).contiguous()
    u = torch.tensor((np.arange(n) + 0.5) / n, dtype=F32, device="cuda")
    tok, _ = api.sample(z, u, temperature=torch.full((n,), T, device="cuda"),
                        top_p=torch.full((n,), p, device="cuda"))
    q = torch.softmax(z[0].double() / T, 0)
    if p < 1:
        v, o = torch.sort(q, descending=True)
        q[o[(v.cumsum(0) - v) >= p]] = 0
        q = q / q.sum()
    got = torch.bincount(tok.long(), minlength=vocab).double()
    assert float((got - n * q).abs().max()) <= 1.01


def test_another_stream_and_a_graph():
    z = logits_of(1, 33, 5000, BF16)
    u = torch.tensor(uniforms(1, 33), device="cuda")
    want = api.sample(z, u)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = api.sample(z, u)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    tokens, conf = torch.empty_like(want[0]), torch.empty_like(want[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        api.sample(z, u, tokens=tokens, conf=conf)
    z.copy_(logits_of(9, 33, 5000, BF16))
    g.replay()
    again = api.sample(z, u)
    assert torch.equal(tokens, again[0]) and not torch.equal(tokens, want[0])


def test_refused_settings():
    n = 8
    z = logits_of(1, n, 500)
    u = torch.full((n,), 0.5, device="cuda")
    nan, inf = float("nan"), float("inf")
    T = torch.tensor([1, -1, nan, inf, 1, 1, 1, 1], device="cuda", dtype=F32)
    p = torch.tensor([.5, .5, .5, .5, 0, nan, .5, .5], device="cuda", dtype=F32)
    m = torch.tensor([0, 0, 0, 0, 0, 0, 1.5, nan], device="cuda", dtype=F32)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    tok, conf = api.sample(z, u, temperature=T, top_p=p, min_p=m, status=status)
    assert B.reflex_read_status(status) == B.REFLEX_EINVAL
    assert int(tok[0]) >= 0 and bool((tok[1:] == -1).all()) and bool((conf[1:] == 0).all())
    with pytest.raises(ValueError):
        api.sample(z.half(), u)
    with pytest.raises(ValueError):
        api.sample(z.t(), u)
    with pytest.raises(ValueError):
        api.sample(z, u[:3])
    with pytest.raises(ValueError):
        api.sample(z, u, top_k=torch.ones(n, device="cuda"))
    with pytest.raises(B.ReflexError):
        api.sample(torch.zeros(1, (1 << 18) + 1, device="cuda"), u[:1])
    tok, conf = api.sample(z[:0], u[:0])
    assert tok.numel() == 0
