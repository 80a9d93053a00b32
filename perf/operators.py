"""The 8-bit serving path of a block-diffusion language model, as cases to time.

A denoising forward in 8 bits quantises its rows, runs the routed experts and
the output head as products of e4m3 codes with one fp32 scale for each block of
128, and samples a token for every masked position; the sampled token's
probability is the confidence that the refinement state takes.  The cases span
one token or one active block (weights and launches are what counts), ordinary
batches and whole batches of sequences, with odd sizes and both storage types.

A case's "op" is the public entry point:
  quantize  api.quantize_fp8: codes and scales of a row for each 128 columns
  linear    api.LinearFp8: rows in bf16 or fp32, weights in 128 x 128 blocks
  experts   api.ExpertsFp8: SwiGLU experts of a routing that the caller holds
  sample    api.sample: temperature, top-k, top-p, min-p from given uniforms
Everything is synthetic and seeded.
"""
import math

import numpy as np
import torch

own = False

BLOCK = 128
DTYPES = dict(bf16=torch.bfloat16, f32=torch.float32)
# layer shapes of the benchmark's two model shapes
MOE = dict(d=2048, E=64, inter=1024)
MINI = dict(d=2048, E=256, inter=512)


def listed():
    return [
        # one active block of 32 tokens before a product: launch latency
        dict(name="quantize_32", op="quantize", rows=32, cols=2048, dtype="bf16"),
        # the benchmark's 32 sequences of 1024 tokens
        dict(name="quantize_32768", op="quantize", rows=32768, cols=2048, dtype="bf16"),
        # one token through a dense layer
        dict(name="linear_1", op="linear", m=1, n=4096, k=2048, dtype="bf16", out="bf16"),
        # the output head on one active block, logits in fp32
        dict(name="head_32", op="linear", m=32, n=65536, k=2048, dtype="bf16", out="f32"),
        # the head on the masked positions of a few sequences, odd row count and vocabulary
        dict(name="head_1000_odd", op="linear", m=999, n=50001, k=2048, dtype="bf16", out="bf16"),
        # the head on a whole serving batch
        dict(name="head_8192", op="linear", m=8192, n=131072, k=2048, dtype="bf16", out="bf16"),
        # one active block with cached keys and values
        dict(name="experts_moe_32", op="experts", tokens=32, k_max=12, residual=True, **MOE),
        # one sequence of 512 + 512 tokens
        dict(name="experts_moe_1024", op="experts", tokens=1024, k_max=12, residual=True, **MOE),
        # the serving batch of the second model shape
        dict(name="experts_mini_8192", op="experts", tokens=8192, k_max=12, residual=False, **MINI),
        # one position, every filter on
        dict(name="sample_1", op="sample", rows=1, vocab=131072, dtype="bf16", filters="all", masked=1.0),
        # one active block, odd vocabulary, fp32 logits, top-k and top-p
        dict(name="sample_32_odd", op="sample", rows=32, vocab=50001, dtype="f32", filters="top_k",
             masked=1.0),
        # a serving batch, half of its positions masked, temperatures and filters row by row
        dict(name="sample_4096", op="sample", rows=4096, vocab=131072, dtype="bf16", filters="mixed",
             masked=0.5),
    ]


def _log(rng, lo, hi):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return n + 1 if n == 3 << 10 else n


def draw(rng):
    op = rng.choice(["quantize", "linear", "linear", "experts", "experts", "sample", "sample"])
    if op == "quantize":
        cols = _log(rng, 1, 8192)
        if rng.random() < 0.6:
            cols = max(1, cols // 128) * 128
        return dict(op=op, rows=_log(rng, 1, max(1, 60000000 // cols)), cols=cols,
                    dtype=rng.choice(["bf16", "bf16", "f32"]))
    if op == "linear":
        k = rng.choice([256, 512, 1024, 2048, 4096, _log(rng, 16, 8000)])
        n = _log(rng, 16, 131072)
        if rng.random() < 0.5:
            n = max(1, n // 64) * 64
        most = min(16384, 2 ** 41 // (n * k), 2 ** 30 // n)
        return dict(op=op, m=_log(rng, 1, most), n=n, k=k,
                    dtype=rng.choice(["bf16", "bf16", "f32"]), out=rng.choice(["bf16", "bf16", "f32"]))
    if op == "experts":
        shape = rng.choice([MOE, MOE, MINI, dict(d=rng.choice([256, 1024, 4096]),
                                                 E=rng.choice([8, 16, 32, 60, 96]),
                                                 inter=rng.choice([128, 192, 512, 768]))])
        return dict(op=op, tokens=_log(rng, 1, 16000), k_max=rng.choice([4, 8, 12]),
                    residual=rng.random() < 0.5, **shape)
    vocab = rng.choice([32000, 65536, 131072, _log(rng, 2, 200000)])
    return dict(op=op, rows=_log(rng, 1, min(8192, 2 ** 27 // vocab)), vocab=vocab,
                dtype=rng.choice(["bf16", "bf16", "f32"]),
                filters=rng.choice(["none", "top_k", "top_p", "min_p", "all", "mixed"]),
                masked=rng.choice([1.0, 1.0, 0.5]))


# ---- inputs -----------------------------------------------------------------
def _normal(g, shape, std, dtype=torch.float32):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)


def _rows(g, rows, cols, dtype):
    """Hidden states: N(0, 1), a few columns ten times as large, as after many layers."""
    x = _normal(g, (rows, cols), 1.0, dtype)
    x[:, 5::301] *= 10
    return x


def _quantize_weights(w):
    """[groups, n, k] to e4m3 codes and fp32 scales of its 128 x 128 blocks, kept by the user."""
    e, n, k = w.shape
    nb, kb = -(-n // BLOCK), -(-k // BLOCK)
    p = torch.zeros((e, nb * BLOCK, kb * BLOCK), device="cuda")
    p[:, :n, :k] = w
    p = p.view(e, nb, BLOCK, kb, BLOCK)
    a = p.abs().amax((2, 4), keepdim=True).clamp(min=2.0 ** -100)
    codes = (p * (448.0 / a)).to(torch.float8_e4m3fn).view(e, nb * BLOCK, kb * BLOCK)
    ld = -(-k // 16) * 16  # rows start on 16-byte boundaries
    out = torch.zeros((e, n, ld), dtype=torch.uint8, device="cuda")
    out[:, :, :k] = codes.view(torch.uint8)[:, :n, :k]
    return out.view(torch.float8_e4m3fn)[:, :, :k], (a / 448.0).view(e, nb, kb)


def _routing(c, seed):
    """Counts in [2, k_max], distinct experts of unequal popularity, weights that sum to 1."""
    g = torch.Generator(device="cuda").manual_seed(seed + 17)
    T, e = c["tokens"], c["E"]
    most = min(c["k_max"], e)
    pop = _normal(g, (1, e), 0.5)
    z = _normal(g, (T, e), 1.0) + pop
    k = torch.randint(min(2, most), most + 1, (T,), generator=g, device="cuda", dtype=torch.int32)
    top = torch.topk(z, most, dim=1)
    used = torch.arange(c["k_max"], device="cuda")[None] < k[:, None]
    ids = torch.full((T, c["k_max"]), -1, dtype=torch.int32, device="cuda")
    ids[:, :most] = top.indices.to(torch.int32)
    ids = torch.where(used, ids, -1)
    alpha = torch.zeros((T, c["k_max"]), device="cuda")
    alpha[:, :most] = torch.softmax(torch.where(used[:, :most], top.values, -math.inf), 1)
    return ids.contiguous(), alpha, k


def _sampling(c, g):
    """Per-row settings: a serving batch mixes greedy, plain and filtered requests."""
    r, f = c["rows"], c["filters"]
    rand = lambda: torch.rand(r, generator=g, device="cuda")  # noqa: E731
    pick = lambda v, dt=torch.float32: torch.tensor(v, dtype=dt, device="cuda")[  # noqa: E731
        (rand() * len(v)).long().clamp(max=len(v) - 1)]
    s = dict(temperature=None, top_k=None, top_p=None, min_p=None, u=rand())
    if f in ("top_k", "all", "mixed"):
        s["top_k"] = pick([20, 50, 200] if f != "mixed" else [0, 0, 50, 1000], torch.int32)
    if f in ("top_k", "top_p", "all", "mixed"):
        s["top_p"] = pick([0.8, 0.9, 0.95] if f != "mixed" else [1.0, 1.0, 0.9, 0.95])
    if f in ("min_p", "all", "mixed"):
        s["min_p"] = pick([0.02, 0.05, 0.1] if f != "mixed" else [0.0, 0.0, 0.05])
    if f != "none":
        s["temperature"] = pick([0.6, 0.8, 1.0, 1.2] if f != "mixed" else [0.0, 0.7, 1.0, 1.0, 1.3])
    return s


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    s = dict(case=c)
    if c["op"] == "quantize":
        s["x"] = _rows(g, c["rows"], c["cols"], DTYPES[c["dtype"]])
    elif c["op"] == "linear":
        s["x"] = _rows(g, c["m"], c["k"], DTYPES[c["dtype"]])
        codes, scales = _quantize_weights(_normal(g, (1, c["n"], c["k"]), 0.02))
        s["w"] = (codes[0], scales[0])
    elif c["op"] == "experts":
        e, d, i = c["E"], c["d"], c["inter"]
        s["hidden"] = _rows(g, c["tokens"], d, torch.bfloat16)
        gu, gu_s = _quantize_weights(_normal(g, (2 * e, i, d), 0.02))  # gate and up by themselves
        s["w_gate_up"] = (gu.view(e, 2 * i, d), gu_s.view(e, 2, *gu_s.shape[1:]))
        s["w_down"] = _quantize_weights(_normal(g, (e, d, i), 0.02))
        s["ids"], s["alpha"], s["k"] = _routing(c, seed)
        s["most"] = int(torch.bincount(s["ids"][s["ids"] >= 0].long(), minlength=e).max())
    else:
        r, v = c["rows"], c["vocab"]
        z = _normal(g, (r, v), 2.0)
        # a few likely tokens a row, from confident rows to undecided ones
        n = min(v, 24)
        at = torch.randint(0, v, (r, 1), generator=g, device="cuda")
        at = (at + torch.arange(n, device="cuda") * (v // n)) % v
        up = torch.rand((r, 1), generator=g, device="cuda") * 12
        z.scatter_add_(1, at, up * torch.rand((r, n), generator=g, device="cuda"))
        s["logits"] = z.to(DTYPES[c["dtype"]])
        s.update(_sampling(c, g))
        s["masked"] = None
        if c["masked"] < 1:
            s["masked"] = (torch.rand(r, generator=g, device="cuda") < c["masked"]).to(torch.uint8)
    if own:
        from paper_2608_01784_gb300 import api
        s["api"] = api
        if c["op"] == "linear":
            s["op"] = api.LinearFp8(*s["w"], max_rows=c["m"], out_dtype=DTYPES[c["out"]])
        elif c["op"] == "experts":
            s["op"] = api.ExpertsFp8(dict(w_gate_up=s["w_gate_up"][0], w_gate_up_scales=s["w_gate_up"][1],
                                          w_down=s["w_down"][0], w_down_scales=s["w_down"][1]),
                                     d=c["d"], E=c["E"], inter=c["inter"], k_max=c["k_max"],
                                     max_tokens=c["tokens"])
    return s


# ---- one pass ---------------------------------------------------------------
def _codes(x):
    """fp32 [.., cols] to e4m3 codes and a scale for each 128 columns."""
    cols, kb = x.shape[-1], -(-x.shape[-1] // BLOCK)
    p = torch.nn.functional.pad(x, (0, kb * BLOCK - cols)).unflatten(-1, (kb, BLOCK))
    a = p.abs().amax(-1, keepdim=True).clamp(min=2.0 ** -100)
    codes = (p * (448.0 / a)).to(torch.float8_e4m3fn)
    return codes.flatten(-2)[..., :cols], (a / 448.0).squeeze(-1)


def _spread(codes, scales, rows=1):
    """The values that codes and scales stand for; a scale covers `rows` x 128 of them."""
    s = scales.repeat_interleave(BLOCK, -1)[..., :codes.shape[-1]]
    if rows > 1:
        s = s.repeat_interleave(rows, -2)[..., :codes.shape[-2], :]
    return codes.float() * s


def _experts(s):
    c = s["case"]
    e, d, i = c["E"], c["d"], c["inter"]
    gu, gus = s["w_gate_up"]
    gate_up = _spread(gu.view(e, 2, i, d), gus, BLOCK).view(e, 2 * i, d)
    down = _spread(*s["w_down"], BLOCK)
    x = _spread(*_codes(s["hidden"].float()))
    # pairs in expert order, `most` rows an expert
    ids = s["ids"].long().flatten()
    ids = torch.where(ids < 0, e, ids)
    order = torch.argsort(ids, stable=True)
    first = torch.searchsorted(ids[order], torch.arange(e + 1, device="cuda"))
    place = torch.empty_like(ids)
    place[order] = torch.arange(ids.numel(), device="cuda") - first[ids[order]]
    used = (ids < e)[:, None]
    row = torch.where(ids < e, ids * s["most"] + place, 0)
    rows = torch.zeros((e * s["most"], d), device="cuda")
    token = torch.arange(ids.numel(), device="cuda") // c["k_max"]
    rows.index_add_(0, row, torch.where(used, x[token], 0.0))
    h = torch.bmm(rows.view(e, -1, d), gate_up.transpose(1, 2))
    g, u = h[..., :i], h[..., i:]
    a = _spread(*_codes(g / (1 + torch.exp(-g)) * u))
    y = torch.bmm(a, down.transpose(1, 2)).view(-1, d)[row]
    y = torch.where(used, y, 0.0) * s["alpha"].flatten()[:, None]
    out = y.view(-1, c["k_max"], d).sum(1)
    if c["residual"]:
        out = out + s["hidden"].float()
    return out.to(torch.bfloat16)


# 2^f on [-1/2, 1/2]: 1 + f (c1 + f (c2 + ...)), Chebyshev interpolation
POLY = (0.6931471824645996, 0.2402234971523285, 0.055503811687231064, 0.00966636836528778,
        0.0013381302123889327)
LOG2E = 1.44269502162933349609375


def _mass(z, m, temperature):
    """Integer weights of the tokens: 2^31 for the largest logit, rounded down."""
    c = torch.clamp(torch.full_like(temperature, LOG2E) / temperature, max=torch.finfo(torch.float32).max)
    t = (z - m) * c[:, None]
    t = torch.where(t > -40, t, -40.0)
    n = torch.round(t)
    f = t - n
    p = torch.full_like(f, POLY[4])
    p = p * f + POLY[3]
    p = p * f + POLY[2]
    p = p * f + POLY[1]
    p = p * f + POLY[0]
    p = p * f + 1.0
    scale = ((n.to(torch.int32) + (127 + 31)) << 23).view(torch.float32)
    return (p * scale).to(torch.int64)


def _sample(s):
    z = s["logits"].float()
    r, v = z.shape
    z = torch.where(z == z, z, -math.inf)
    m = z.amax(1, keepdim=True)
    z = torch.where(m == math.inf, torch.where(z == math.inf, 0.0, -math.inf), z)
    m = torch.where(m == math.inf, 0.0, m)
    e = torch.exp(z - m)
    whole = lambda x: torch.full((r,), x, device="cuda")  # noqa: E731
    temp = s["temperature"] if s["temperature"] is not None else whole(1.0)
    greedy = temp == 0
    temp = torch.where(greedy, 1.0, temp)
    rank_z, order = torch.sort(z, dim=1, descending=True, stable=True)
    w = _mass(rank_z, m, temp)
    kept = torch.ones_like(w, dtype=torch.bool)
    if s["top_k"] is not None:
        k = torch.where(s["top_k"] > 0, s["top_k"], v)
        kept = torch.arange(v, device="cuda")[None] < k[:, None]
    if s["top_p"] is not None:
        p = torch.where(s["top_p"] < 1, s["top_p"], 2.0).double()
        w_k = torch.where(kept, w, 0)
        before = w_k.cumsum(1) - w_k
        kept = kept & (before.double() < (p * w_k.sum(1).double())[:, None])
    if s["min_p"] is not None:
        kept = kept & (w >= torch.ceil(s["min_p"].double() * 2.0 ** 31)[:, None])
    w = torch.where(kept, w, 0)
    w = torch.zeros_like(w).scatter_(1, order, w)  # back in index order
    total = w.sum(1).double()
    over = w.cumsum(1).double() > (s["u"].double() * total)[:, None]
    token = torch.where(greedy, order[:, 0], over.to(torch.uint8).argmax(1))
    conf = e.gather(1, token[:, None])[:, 0] / e.sum(1)
    alive = m[:, 0] > -math.inf
    if s["masked"] is not None:
        alive = alive & (s["masked"] != 0)
    return dict(tokens=torch.where(alive, token, -1).to(torch.int32), conf=torch.where(alive, conf, 0.0))


def run(state):
    s = state
    op = s["case"]["op"]
    if own:
        if op == "quantize":
            return s["api"].quantize_fp8(s["x"])
        if op == "linear":
            return s["op"].forward(s["x"])
        if op == "experts":
            return s["op"].forward(s["hidden"], s["ids"], s["alpha"], s["k"],
                                   residual=s["case"]["residual"])
        tokens, conf = s["api"].sample(s["logits"], s["u"], temperature=s["temperature"],
                                       top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"],
                                       masked=s["masked"])
        return dict(tokens=tokens, conf=conf)
    if op == "quantize":
        return _codes(s["x"].float())
    if op == "linear":
        out = _spread(*_codes(s["x"].float())) @ _spread(*s["w"], BLOCK).T
        return out.to(DTYPES[s["case"]["out"]])
    return _experts(s) if op == "experts" else _sample(s)


# ---- what a pass cannot do without ------------------------------------------
def work(case):
    c = case
    if c["op"] == "quantize":
        es = 2 if c["dtype"] == "bf16" else 4
        n = c["rows"] * c["cols"]
        return dict(bytes=n * (es + 1) + 4 * c["rows"] * -(-c["cols"] // BLOCK), flops=0)
    if c["op"] == "linear":
        m, n, k = c["m"], c["n"], c["k"]
        es, eo = (2 if c[t] == "bf16" else 4 for t in ("dtype", "out"))
        return dict(bytes=m * k * es + n * k + m * n * eo, flops=2 * m * n * k)
    if c["op"] == "experts":
        T, e, d, i = c["tokens"], c["E"], c["d"], c["inter"]
        most = min(c["k_max"], e)
        pairs = T * (min(2, most) + most) / 2
        touched = e * (1 - (1 - 1 / e) ** pairs)
        return dict(bytes=touched * 3 * d * i + 2 * T * d * 2 + T * c["k_max"] * 8,
                    flops=6 * pairs * d * i)
    es = 2 if c["dtype"] == "bf16" else 4
    return dict(bytes=max(1, c["rows"] * c["masked"]) * (c["vocab"] * es + 28),
                flops=20 * c["rows"] * c["masked"] * c["vocab"])


# ---- the same in 64 bits ----------------------------------------------------
def _e4m3_64(x):
    """Nearest e4m3 value (ties to even) of 64-bit numbers of at most 448 and a little."""
    q = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / q) * q


def _codes64(x):
    cols, kb = x.shape[-1], -(-x.shape[-1] // BLOCK)
    p = torch.zeros((*x.shape[:-1], kb * BLOCK), dtype=torch.float64, device="cuda")
    p[..., :cols] = x
    p = p.view(*x.shape[:-1], kb, BLOCK)
    a = torch.clamp(p.abs().amax(-1, keepdim=True), min=2.0 ** -100)
    return _e4m3_64(p * 448 / a), a / 448


def _rows64(x):
    codes, scale = _codes64(x)
    return (codes * scale).flatten(-2)[..., :x.shape[-1]]


def _weights64(codes, scales):
    n, k = codes.shape
    r, c = torch.arange(n, device="cuda") // BLOCK, torch.arange(k, device="cuda") // BLOCK
    return codes.double() * scales.double()[r][:, c]


def _experts64(c, s):
    x = _rows64(s["hidden"].double())
    out = s["hidden"].double() if c["residual"] else torch.zeros_like(x)
    out, i = out.clone(), c["inter"]
    for e in range(c["E"]):
        t, j = torch.nonzero(s["ids"] == e, as_tuple=True)
        if not t.numel():
            continue
        gu, gus = s["w_gate_up"][0][e], s["w_gate_up"][1][e]
        g = x[t] @ _weights64(gu[:i], gus[0]).T
        a = g * torch.sigmoid(g) * (x[t] @ _weights64(gu[i:], gus[1]).T)
        y = _rows64(a) @ _weights64(s["w_down"][0][e], s["w_down"][1][e]).T
        out.index_add_(0, t, s["alpha"][t, j].double()[:, None] * y)
    return out


def _sample64(s):
    """Confidence of the token that inverting the kept distribution gives, row by row."""
    z = s["logits"].double().cpu().numpy()
    host = lambda x, rows, other: (np.full(rows, other) if x is None else x.cpu().numpy())  # noqa: E731
    r, v = z.shape
    temp, top_k = host(s["temperature"], r, 1.0), host(s["top_k"], r, 0)
    top_p, min_p = host(s["top_p"], r, 1.0), host(s["min_p"], r, 0.0)
    live, u = host(s["masked"], r, 1), s["u"].double().cpu().numpy()
    conf = np.zeros(r)
    for i in range(r):
        if not live[i]:
            continue
        row = z[i]
        p = np.exp(row - row.max())
        if temp[i] == 0:
            tok = int(row.argmax())
        else:
            w = np.exp((row - row.max()) / np.float64(temp[i]))
            keep = w >= min_p[i]
            if top_k[i] > 0 or top_p[i] < 1:
                order = np.argsort(-row, kind="stable")
                q = w[order]
                if top_k[i] > 0:
                    q[top_k[i]:] = 0
                before = np.cumsum(q) - q
                cut = (q > 0) & ((before < top_p[i] * q.sum()) | (top_p[i] >= 1))
                keep[order[~cut]] = False
            run_sum = np.cumsum(np.where(keep, w, 0.0))
            tok = int(np.searchsorted(run_sum, u[i] * run_sum[-1], side="right"))
        conf[i] = p[tok] / p.sum()
    return torch.from_numpy(conf)


def exact(case, seed):
    c = case
    # 64-bit products run at about 1 TFLOP/s here, the rows of a sample at 10 million logits a second
    if work(c)["flops"] > (1e9 if c["op"] == "sample" else 5e12):
        return None
    s = prepare(c, seed)
    if c["op"] == "quantize":
        codes, scale = _codes64(s["x"].double())
        return codes.flatten(-2)[..., :c["cols"]], scale.squeeze(-1)
    if c["op"] == "linear":
        return _rows64(s["x"].double()) @ _weights64(*s["w"]).T
    if c["op"] == "experts":
        return _experts64(c, s)
    return dict(tokens=None, conf=_sample64(s))
