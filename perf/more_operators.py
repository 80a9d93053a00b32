"""What stands around a block's experts and behind the last layer, as cases to time.

A block of a diffusion language model is more than its experts: the residual
stream is normalised in front of it, its output normalised, gated and scaled
back into the stream; the tokens are laid out by expert and summed back with
their router weights; and behind the last layer, tuning or scoring a model asks
for the cross entropy of the output head on the masked positions.  Each of the
three has its gradient.  The cases span one token or one active block (launches
count), ordinary batches and the benchmark's 32 sequences of 1024 tokens, with
odd sizes and both storage types.

A case's "op" and "way" name the public entry points:
  norm  forward   api.block_norm: o = h + s g norm(y), n = norm(o)
        gradient  api.block_norm_backward
  sort  forward   api.expert_plan, api.expert_rows: tokens in expert order
        gradient  api.expert_rows_backward
  back  forward   api.expert_combine: the weighted sum in token order, with a residual
        gradient  api.expert_combine_backward
  loss  forward   api.head_loss: cross entropy of a vocabulary head, no logits kept
        gradient  api.head_loss, then api.head_loss_backward (a tuning step of the head)
Everything is synthetic and seeded.
"""
import math

import torch

own = False

DTYPES = dict(bf16=torch.bfloat16, f32=torch.float32)
EPS = 1e-6


def listed():
    return [
        # one active block of 32 tokens between two layers: launch latency
        dict(name="norm_32", op="norm", way="forward", rows=32, d=2048, dtype="bf16", after=True,
             gate="channel", before=True),
        # the benchmark's 32 sequences of 1024 tokens
        dict(name="norm_32768", op="norm", way="forward", rows=32768, d=2048, dtype="bf16", after=True,
             gate="channel", before=True),
        # its gradient in a tuning step
        dict(name="norm_grad_32768", op="norm", way="gradient", rows=32768, d=2048, dtype="bf16",
             after=True, gate="channel", before=True),
        # an odd batch in fp32, modulated token by token
        dict(name="norm_grad_odd", op="norm", way="gradient", rows=1999, d=1001, dtype="f32", after=True,
             gate="token", before=True),
        # one active block to its experts: launch latency
        dict(name="sort_32", op="sort", way="forward", tokens=32, d=2048, E=64, k_max=12, dtype="bf16"),
        # the benchmark's batch to its experts
        dict(name="sort_32768", op="sort", way="forward", tokens=32768, d=2048, E=64, k_max=12,
             dtype="bf16"),
        # and back, many small experts
        dict(name="back_8192", op="back", way="forward", tokens=8192, d=2048, E=256, k_max=12, dtype="bf16"),
        # the gradient of the way back, with the router weights'
        dict(name="back_grad_8192", op="back", way="gradient", tokens=8192, d=2048, E=64, k_max=12,
             dtype="bf16"),
        # scoring one active block
        dict(name="loss_32", op="loss", way="forward", rows=32, vocab=65536, k=2048, masked=1.0),
        # scoring a batch of sequences, half of it masked
        dict(name="loss_8192", op="loss", way="forward", rows=8192, vocab=131072, k=2048, masked=0.5),
        # a step on the masked positions of a few sequences, odd row count and vocabulary
        dict(name="loss_grad_999_odd", op="loss", way="gradient", rows=999, vocab=50001, k=2048, masked=1.0),
        # a step on a whole batch
        dict(name="loss_grad_8192", op="loss", way="gradient", rows=8192, vocab=131072, k=2048, masked=1.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm", "sort", "back", "back", "loss", "loss"])
    way = rng.choice(["forward", "gradient"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "norm":
        d = rng.choice([256, 1024, 2048, 4096, _log(rng, 1, 16384)])
        after, before = rng.choice([(True, True), (True, True), (False, True), (True, False)])
        return dict(op=op, way=way, rows=_log(rng, 1, max(1, 2 ** 26 // d)), d=d, dtype=dtype, after=after,
                    gate=rng.choice(["none", "channel", "token"]), before=before)
    if op in ("sort", "back"):
        d = rng.choice([256, 1024, 2048, 4096, _log(rng, 1, 8192)])
        k_max = rng.choice([1, 4, 8, 12, 12])
        return dict(op=op, way=way, tokens=_log(rng, 1, max(1, 2 ** 29 // (d * k_max))), d=d,
                    E=rng.choice([8, 60, 64, 64, 256]), k_max=k_max, dtype=dtype)
    k = rng.choice([256, 512, 1024, 2048, 2048, 4096, _log(rng, 8, 5000)])
    vocab = rng.choice([32000, 65536, 131072, _log(rng, 2, 200000)])
    most = min(16384, 2 ** 41 // (k * vocab), 2 ** 30 // vocab)
    return dict(op=op, way=way, rows=_log(rng, 1, most), vocab=vocab, k=k, masked=rng.choice([1.0, 0.75, 0.5]))


# ---- inputs -----------------------------------------------------------------
def _normal(g, shape, std, dtype=torch.float32):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)


def _stream(g, rows, cols, dtype):
    """A residual stream: N(0, 1), a few columns ten times as large, as after many layers."""
    x = _normal(g, (rows, cols), 1.0, dtype)
    x[:, 5::301] *= 10
    return x


def _routing(c, g):
    """Counts in [2, k_max], distinct experts of unequal popularity, weights that sum to 1."""
    T, e, most = c["tokens"], c["E"], min(c["k_max"], c["E"])
    z = _normal(g, (T, e), 1.0) + _normal(g, (1, e), 0.5)
    k = torch.randint(min(2, most), most + 1, (T,), generator=g, device="cuda", dtype=torch.int32)
    top = torch.topk(z, most, dim=1)
    used = torch.arange(most, device="cuda")[None] < k[:, None]
    ids = torch.full((T, c["k_max"]), -1, dtype=torch.int32, device="cuda")
    ids[:, :most] = torch.where(used, top.indices.to(torch.int32), -1)
    alpha = torch.zeros((T, c["k_max"]), device="cuda")
    alpha[:, :most] = torch.softmax(torch.where(used, top.values, -math.inf), 1)
    return ids, alpha


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    s = dict(case=c)
    if c["op"] == "norm":
        dt, T, d = DTYPES[c["dtype"]], c["rows"], c["d"]
        s["h"], s["y"] = _stream(g, T, d, dt), _normal(g, (T, d), 0.5, dt)
        weight = lambda: (1 + _normal(g, (d,), 0.1)).to(dt)  # noqa: E731
        s["opt"] = dict(w_after=weight() if c["after"] else None, w_before=weight() if c["before"] else None,
                        gate={"none": None, "channel": _normal(g, (d,), 0.5, dt),
                              "token": _normal(g, (T, d), 0.5, dt)}[c["gate"]],
                        scale=0.7, eps=EPS)
        if c["way"] == "gradient":
            s["d_out"] = _normal(g, (T, d), 1e-3, dt)
            s["d_norm"] = _normal(g, (T, d), 1e-3, dt) if c["before"] else None
    elif c["op"] in ("sort", "back"):
        dt, T, d = DTYPES[c["dtype"]], c["tokens"], c["d"]
        s["ids"], s["alpha"] = _routing(c, g)
        cap = T * c["k_max"]
        if c["op"] == "sort" and c["way"] == "forward":
            s["x"] = _stream(g, T, d, dt)
        else:  # the experts' outputs, or the gradient of the rows
            s["rows"] = _normal(g, (cap, d), 0.5, dt)
        if c["op"] == "back":
            s["x"] = _stream(g, T, d, dt)  # the residual, or the gradient of the output
        # buffers of the whole capacity that a program keeps: rows behind the last pair stay as they are
        if (c["op"] == "sort") == (c["way"] == "forward"):
            s["to"] = torch.zeros((cap, d), dtype=dt, device="cuda")
    else:
        M, v, k = c["rows"], c["vocab"], c["k"]
        ld = -(-k // 8) * 8  # rows start on 16-byte boundaries
        s["w"] = _normal(g, (v, ld), 2.0 / math.sqrt(k), torch.bfloat16)[:, :k]
        t = torch.randint(0, v, (M,), generator=g, device="cuda", dtype=torch.int32)
        h = _normal(g, (M, ld), 1.0)
        # from rows that know nothing of their token to rows that are sure of it
        sure = torch.rand((M, 1), generator=g, device="cuda") * 3
        h[:, :k] += sure * s["w"][t.long()].float()
        s["hidden"] = h.to(torch.bfloat16)[:, :k]
        live = torch.rand(M, generator=g, device="cuda") < c["masked"]
        s["targets"] = torch.where(live, t, -1)
        # the weight of a position falls with the share of masked ones in its sequence
        share = torch.rand(M, generator=g, device="cuda") * 0.8 + 0.2
        s["grad"] = torch.where(live, 1 / (share * M), 0.0)
    if own:
        from paper_2608_01784_gb300 import api
        s["api"] = api
        if c["op"] == "back" or (c["op"] == "sort" and c["way"] == "gradient"):
            s["plan"] = api.expert_plan(s["ids"], E=c["E"])
    return s


# ---- one pass ---------------------------------------------------------------
def _rms(x):
    return 1 / torch.sqrt((x * x).mean(1, keepdim=True) + EPS)


def _norm(s):
    """The formulas in 32 bits: outputs, or the gradients of all inputs."""
    c, opt = s["case"], s["opt"]
    dt = DTYPES[c["dtype"]]
    f = lambda x: None if x is None else x.float()  # noqa: E731
    h, y, wa, wb, gate, scale = (f(s["h"]), f(s["y"]), f(opt["w_after"]), f(opt["w_before"]),
                                 f(opt["gate"]), opt["scale"])
    ry = _rms(y)
    yh = y * ry
    a = y if wa is None else yh * wa
    o = h + scale * (a if gate is None else gate * a)
    ro = _rms(o)
    if c["way"] == "forward":
        return dict(out=o.to(dt), norm=None if wb is None else (o * ro * wb).to(dt))
    do, dn = f(s["d_out"]), f(s["d_norm"])
    out = dict(w_after=None, w_before=None, gate=None)
    if wb is not None:
        oh, v = o * ro, dn * wb
        do = do + ro * (v - oh * (v * oh).mean(1, keepdim=True))
        out["w_before"] = (dn * oh).sum(0).to(dt)
    out["h"] = do.to(dt)
    b = scale * do
    if gate is not None:
        dg = b * a
        out["gate"] = (dg.sum(0) if gate.dim() == 1 else dg).to(dt)
        b = b * gate
    if wa is not None:
        out["w_after"] = (b * yh).sum(0).to(dt)
        u = b * wa
        b = ry * (u - yh * (u * yh).mean(1, keepdim=True))
    out["y"] = b.to(dt)
    return out


def _plan(s):
    """Pairs in order of (expert, token, slot): the row of each, -1 for unused slots."""
    c = s["case"]
    ids = s["ids"].long().flatten()
    used = ids >= 0
    key = torch.where(used, ids, c["E"])
    order = torch.argsort(key, stable=True)
    row = torch.empty_like(order)
    row[order] = torch.arange(order.numel(), device="cuda")
    row = torch.where(used, row, -1)
    offsets = torch.searchsorted(key[order], torch.arange(c["E"] + 1, device="cuda"))
    return row.view(s["ids"].shape), offsets


def _pairs(s):
    c = s["case"]
    dt = DTYPES[c["dtype"]]
    row, offsets = _plan(s)
    if (c["op"] == "sort") == (c["way"] == "forward"):
        # to expert order: a spare row behind the others takes the unused slots
        to = torch.zeros((s["to"].shape[0] + 1, c["d"]), device="cuda")
        at = torch.where(row >= 0, row, s["to"].shape[0])
        for j in range(c["k_max"]):
            x = s["x"].float()
            to[at[:, j]] = x if c["op"] == "sort" else x * s["alpha"][:, j, None]
        to = to[:-1].to(dt)
        if c["op"] == "sort":
            return dict(row_of=row.to(torch.int32), offsets=offsets.to(torch.int32), rows=to)
        d_alpha = [(s["x"].float() * s["rows"][row[:, j].clamp(min=0)].float()).sum(1) for j in range(c["k_max"])]
        return dict(rows=to, alpha=torch.where(row >= 0, torch.stack(d_alpha, 1), 0.0))
    out = torch.zeros((c["tokens"], c["d"]), device="cuda")
    for j in range(c["k_max"]):
        y = s["rows"][row[:, j].clamp(min=0)].float()
        if c["op"] == "back":
            y = y * s["alpha"][:, j, None]
        out = out + torch.where(row[:, j, None] >= 0, y, 0.0)
    if c["op"] == "back":
        out = out + s["x"].float()
    return out.to(dt)


def _loss(s):
    h, w, live = s["hidden"].float(), s["w"].float(), s["targets"] >= 0
    z = h @ w.T
    m = z.amax(1, keepdim=True)
    lse = m + torch.log(torch.exp(z - m).sum(1, keepdim=True))
    t = s["targets"].long().clamp(min=0)[:, None]
    zero = torch.zeros((), device="cuda")
    out = dict(loss=torch.where(live, (lse - z.gather(1, t))[:, 0], zero), lse=torch.where(live, lse[:, 0], zero))
    if s["case"]["way"] == "gradient":
        g = torch.exp(z - lse)
        del z
        g.scatter_add_(1, t, torch.full(t.shape, -1.0, device="cuda"))
        g *= torch.where(live, s["grad"], zero)[:, None]
        out["hidden"] = (g @ w).to(torch.bfloat16)
        out["weight"] = (g.T @ h).to(torch.bfloat16)
    return out


def run(state):
    s = state
    c = s["case"]
    op, way = c["op"], c["way"]
    if not own:
        return _norm(s) if op == "norm" else _loss(s) if op == "loss" else _pairs(s)
    api = s["api"]
    if op == "norm":
        if way == "forward":
            out, norm = api.block_norm(s["h"], s["y"], **s["opt"])
            return dict(out=out, norm=norm)
        return api.block_norm_backward(s["h"], s["y"], s["d_out"], s["d_norm"], **s["opt"])
    if op == "sort":
        if way == "forward":
            plan = api.expert_plan(s["ids"], E=c["E"])
            rows = api.expert_rows(s["x"], plan, rows=s["to"])
            return dict(row_of=plan.row_of, offsets=plan.offsets, rows=rows)
        return api.expert_rows_backward(s["rows"], s["plan"])
    if op == "back":
        if way == "forward":
            return api.expert_combine(s["rows"], s["alpha"], s["plan"], residual=s["x"])
        rows, alpha = api.expert_combine_backward(s["x"], s["rows"], s["alpha"], s["plan"], d_rows=s["to"])
        return dict(rows=rows, alpha=alpha)
    loss, lse = api.head_loss(s["hidden"], s["w"], s["targets"])
    if way == "forward":
        return dict(loss=loss, lse=lse)
    hidden, weight = api.head_loss_backward(s["hidden"], s["w"], s["targets"], lse, s["grad"])
    return dict(loss=loss, lse=lse, hidden=hidden, weight=weight)


# ---- what a pass cannot do without ------------------------------------------
def work(case):
    c = case
    grad = c["way"] == "gradient"
    if c["op"] == "norm":
        es = 2 if c["dtype"] == "bf16" else 4
        n = (5 if grad else 3) + c["before"]  # h, y, out, norm; gradients: h, y, Dout, Dnorm, Dh, Dy
        if c["gate"] == "token":
            n += 2 if grad else 1
        return dict(bytes=n * c["rows"] * c["d"] * es, flops=(30 if grad else 10) * c["rows"] * c["d"])
    if c["op"] in ("sort", "back"):
        es = 2 if c["dtype"] == "bf16" else 4
        T, most = c["tokens"], min(c["k_max"], c["E"])
        pairs = T * (min(2, most) + most) / 2
        n = pairs + T  # rows on one side, tokens on the other
        if c["op"] == "back":
            n += pairs if grad else T
        return dict(bytes=n * c["d"] * es + 8 * T * c["k_max"],
                    flops=(0 if c["op"] == "sort" and not grad else 2 * pairs * c["d"] * (2 if grad else 1)))
    m, v, k = max(1, c["rows"] * c["masked"]), c["vocab"], c["k"]
    return dict(bytes=2 * (m * k + v * k) * (2 if grad else 1) + 16 * c["rows"],
                flops=(6 if grad else 2) * m * v * k)


# ---- the same in 64 bits ----------------------------------------------------
def _norm64(c, s):
    names = ("h", "y", "w_after", "w_before", "gate")
    x = {n: s[n] if n in s else s["opt"][n] for n in names}
    x = {n: None if t is None else t.double().requires_grad_(c["way"] == "gradient") for n, t in x.items()}
    norm = lambda t, w: t * torch.rsqrt(t.square().sum(1) / c["d"] + s["opt"]["eps"])[:, None] * w  # noqa: E731
    b = x["y"] if x["w_after"] is None else norm(x["y"], x["w_after"])
    if x["gate"] is not None:
        b = b * x["gate"]
    o = x["h"] + b * s["opt"]["scale"]
    n = None if x["w_before"] is None else norm(o, x["w_before"])
    if c["way"] == "forward":
        return dict(out=o, norm=n)
    total = (o * s["d_out"].double()).sum()
    if n is not None:
        total = total + (n * s["d_norm"].double()).sum()
    given = [m for m in names if x[m] is not None]
    grads = dict(zip(given, torch.autograd.grad(total, [x[m] for m in given])))
    return {m: grads.get(m) for m in ("w_after", "w_before", "gate", "h", "y")}


def _pairs64(c, s):
    ids = s["ids"]
    t, j = torch.nonzero(ids >= 0, as_tuple=True)  # by token and slot
    e = ids[t, j]
    order = torch.argsort(e, stable=True)
    t, j = t[order], j[order]  # pair number r belongs to token t[r], slot j[r]
    n = t.numel()
    if (c["op"] == "sort") == (c["way"] == "forward"):
        to = torch.zeros(s["to"].shape, dtype=torch.float64, device="cuda")
        x = s["x"].double()
        if c["op"] == "sort":
            to[:n] = x[t]
            return dict(row_of=None, offsets=None, rows=to)
        to[:n] = x[t] * s["alpha"].double()[t, j][:, None]
        alpha = torch.zeros(ids.shape, dtype=torch.float64, device="cuda")
        alpha[t, j] = torch.einsum("rd,rd->r", x[t], s["rows"][:n].double())
        return dict(rows=to, alpha=alpha)
    y = s["rows"][:n].double()
    if c["op"] == "sort":
        return torch.zeros((c["tokens"], c["d"]), dtype=torch.float64, device="cuda").index_add_(0, t, y)
    return s["x"].double().index_add_(0, t, y * s["alpha"].double()[t, j][:, None])


def _loss64(c, s):
    w, M = s["w"].double(), c["rows"]
    zeros = lambda *n: torch.zeros(n, dtype=torch.float64, device="cuda")  # noqa: E731
    out = dict(loss=zeros(M), lse=zeros(M))
    if c["way"] == "gradient":
        out.update(hidden=zeros(M, c["k"]), weight=zeros(c["vocab"], c["k"]))
    rows = torch.nonzero(s["targets"] >= 0)[:, 0]
    for i in rows.split(max(1, 2 ** 28 // c["vocab"])):
        h, t = s["hidden"][i].double(), s["targets"][i].long()
        logp = torch.log_softmax(h @ w.T, 1)
        at = torch.arange(i.numel(), device="cuda")
        out["loss"][i] = -logp[at, t]
        out["lse"][i] = (h * w[t]).sum(1) - logp[at, t]
        if c["way"] == "gradient":
            p = logp.exp_()
            p[at, t] -= 1
            p *= s["grad"][i].double()[:, None]
            out["hidden"][i] = p @ w
            out["weight"] += p.T @ h
    return out


def exact(case, seed):
    c = case
    if c["op"] == "loss" and work(c)["flops"] > 5e12:  # 64-bit products run at about 1 TFLOP/s here
        return None
    s = prepare(c, seed)
    return _norm64(c, s) if c["op"] == "norm" else _loss64(c, s) if c["op"] == "loss" else _pairs64(c, s)
