"""Cuts anywhere in a row: top-p next to 1, top-k of thousands.  The tokens are the
definition's, and a cut far down costs no several walks over the row more than a near
one."""
import numpy as np
import pytest
import torch

from paper_2608_01784_gb300 import api
from tests.test_gpu_sample import BF16, F32, check, logits_of, uniforms

pytestmark = pytest.mark.gpu
F = np.float32


def peaked(rows, vocab, dtype, mass=22.0):
    z = logits_of(rows, rows, vocab, F32)
    z[torch.arange(rows), torch.arange(rows) * 31 % vocab] = mass
    return z.to(dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,vocab", [(12, 3001), (12, 50001), (90, 60001)])
@pytest.mark.parametrize("kind", ["spread", "peaked", "ties", "tails"])
def test_top_p_next_to_one(rows, vocab, dtype, kind):
    if kind == "spread":
        z = logits_of(3, rows, vocab, dtype)
    elif kind == "peaked":
        z = peaked(rows, vocab, dtype, 13.0)
    elif kind == "ties":
        z = (torch.arange(rows * vocab, device="cuda").view(rows, vocab) % 5).float().to(dtype)
    else:  # weights down to the last that count, and below
        z = torch.linspace(-40, 0, vocab, device="cuda").expand(rows, vocab).contiguous().to(dtype)
    p = np.resize(np.array([0.98, 0.985, 0.9881, 0.99, 0.995, 0.9971, 0.999, 0.9999, 0.99999,
                            1 - 2.0 ** -24, 0.5, 1e-6], F), rows)
    check(z, uniforms(1, rows), p=p)
    check(z, uniforms(2, rows), p=p, T=np.full(rows, 0.6, F))
    check(z, uniforms(3, rows), p=p, k=np.full(rows, 2000), min_p=np.full(rows, 1e-4, F))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_top_k_of_thousands(dtype):
    rows, vocab = 90, 70001
    k = np.resize(np.array([2000, 2500, 2560, 2561, 3000, 3500, 4000, 4374, 4376, 10240, 10241,
                            30000, 70000, 70001, 70002]), rows)
    z = logits_of(7, rows, vocab, dtype)
    check(z, uniforms(4, rows), k=k)
    check(z, uniforms(5, rows), k=k, p=np.full(rows, 0.97, F))


def us(run, n=4):
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(n):
            run()
    best = float("inf")
    for _ in range(5):
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        graph.replay()
        b.record()
        torch.cuda.synchronize()
        best = min(best, a.elapsed_time(b) * 1e3 / n)
    return best


@pytest.mark.parametrize("kind", ["spread", "peaked"])
def test_far_cuts_cost_no_walk_over_every_token(kind):
    """304 rows of 131072: five to six times as long where the row is searched whole."""
    rows, vocab = 304, 131072
    z = logits_of(1, rows, vocab, BF16) if kind == "spread" else peaked(rows, vocab, BF16)
    u = torch.tensor(uniforms(1, rows), device="cuda")
    tokens = torch.empty(rows, dtype=torch.int32, device="cuda")
    conf = torch.empty(rows, device="cuda")

    def time(**settings):
        kw = {n: torch.full((rows,), v, dtype=torch.int32 if n == "top_k" else F32, device="cuda")
              for n, v in settings.items()}
        return us(lambda: api.sample(z, u, tokens=tokens, conf=conf, **kw))
    near = time(top_p=0.9)
    for p in (0.985, 0.99, 0.999, 0.9999):
        assert time(top_p=p) <= 2 * near, (p, near)


@pytest.mark.parametrize("kind", ["spread", "peaked"])
def test_top_k_of_thousands_costs_no_walk_over_every_token(kind):
    """The same rows: six times as long where the list cannot hold what is asked for."""
    rows, vocab = 304, 131072
    z = logits_of(1, rows, vocab, BF16) if kind == "spread" else peaked(rows, vocab, BF16)
    u = torch.tensor(uniforms(1, rows), device="cuda")
    tokens = torch.empty(rows, dtype=torch.int32, device="cuda")
    conf = torch.empty(rows, device="cuda")

    def time(k):
        k = torch.full((rows,), k, dtype=torch.int32, device="cuda")
        return us(lambda: api.sample(z, u, tokens=tokens, conf=conf, top_k=k))
    near = time(9000)
    for k in (2000, 2560, 3000, 3500, 5000, 8000):
        assert time(k) <= 2 * near, (k, near)
