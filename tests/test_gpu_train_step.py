"""A training step of a small masked model from the calls together: norms around two
blocks of experts, tokens to the experts and back, the loss of the head on the masked
positions, and the gradients all the way down, against autograd in 64 bits.

The experts' products are torch's (fp32 matrices, without TF32).  Tolerances: every
stored tensor is bf16, a step off by 2^-8 at most, and a gradient goes through about 16
of them on its way to the front; rounding errors of independent elements add like
squares over a tensor, so the relative error in the Euclidean norm is below 4 times one
step's 2^-8, twice that for a factor that cancellation takes: SMOOTH.

What has gone back through a ReLU has one error more.  A unit whose input e perturbs
across 0 passes a gradient where it should not, or none where it should.  Inputs are
about normal, of size 1, and off by E|e| <= 2^-8 of it (the roundings of x and of the
stream in front of it), so a share of 2 phi(0) E|e| = 0.8 * 2^-8 of the units flip.  All of
a flipped unit's gradient is wrong; half of the units are active, so the squared error
is up to 2 * 0.8 * 2^-8 of the squared gradient a ReLU, 0.0125 for two, the error 0.112."""
import pytest
import torch

from paper_2608_01784_gb300 import api

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
T, D, INTER, E, K, VOCAB = 300, 96, 64, 6, 3, 701
EPS = 1e-6
SMOOTH = 8 * 2.0 ** -8
THROUGH_RELU = SMOOTH + 0.112


def make(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def draw(*shape, std=1.0, mean=0.0):
        return (torch.randn(*shape, generator=g, device="cuda") * std + mean).to(BF16)
    layers = [dict(w1=draw(E, INTER, D, std=D ** -0.5), w2=draw(E, D, INTER, std=INTER ** -0.5),
                   w_before=draw(D, std=0.1, mean=1), w_after=draw(D, std=0.1, mean=1),
                   gate=draw(D, std=0.1, mean=1)) for _ in range(2)]
    ids = torch.stack([torch.randperm(E, generator=g, device="cuda")[:K] for _ in range(T)]).int()
    used = torch.arange(K, device="cuda")[None] < torch.randint(1, K + 1, (T, 1), generator=g,
                                                                device="cuda")
    ids = torch.where(used, ids, -1)
    alpha = torch.where(used, torch.rand(T, K, generator=g, device="cuda"), 0.0)
    targets = torch.randint(0, VOCAB, (T,), generator=g, device="cuda", dtype=torch.int32)
    targets[torch.rand(T, generator=g, device="cuda") < 0.4] = -1
    return dict(layers=layers, ids=ids, alpha=alpha, targets=targets, hidden=draw(T, D),
                final=draw(D, std=0.1, mean=1), head=draw(VOCAB, D, std=2 * D ** -0.5))


def experts(rows, offsets, w, each):
    """each(rows of an expert, its weights) for every expert, in place of empty rows none."""
    out = torch.zeros_like(rows)
    for e in range(E):
        lo, hi = int(offsets[e]), int(offsets[e + 1])
        if hi > lo:
            out[lo:hi] = each(rows[lo:hi], w, e)
    return out


def up_down(x, w, e):
    a = torch.relu(x.float() @ w["w1"][e].float().T).to(BF16)
    return (a.float() @ w["w2"][e].float().T).to(BF16)


def step(m):
    """Loss and gradients from the framework's calls."""
    live = (m["targets"] >= 0).sum()
    plan = api.expert_plan(m["ids"], E=E)
    offsets = plan.offsets.tolist()
    L = m["layers"]
    h, x = api.block_norm(m["hidden"], w_before=L[0]["w_before"], eps=EPS)
    kept = []
    for i, w in enumerate(L):
        rows = api.expert_rows(x, plan)
        y_rows = experts(rows, offsets, w, up_down)
        y = api.expert_combine(y_rows, m["alpha"], plan)
        after = L[i + 1]["w_before"] if i + 1 < len(L) else m["final"]
        opt = dict(w_after=w["w_after"], gate=w["gate"], w_before=after, scale=0.7, eps=EPS)
        kept.append((h, y, rows, y_rows, opt))
        h, x = api.block_norm(h, y, **opt)
    loss, lse = api.head_loss(x, m["head"], m["targets"])
    grad = torch.where(m["targets"] >= 0, 1.0 / live, 0.0).float()
    d_x, d_head = api.head_loss_backward(x, m["head"], m["targets"], lse, grad)
    got = dict(loss=loss.double().sum() / live, head=d_head)
    d_h = None
    for i in reversed(range(len(L))):
        h, y, rows, y_rows, opt = kept[i]
        g = api.block_norm_backward(h, y, d_h, d_x, **opt)
        got.update({f"w_after{i}": g["w_after"], f"gate{i}": g["gate"],
                    f"w_before{i + 1}": g["w_before"]})
        d_h = g["h"]
        d_rows, d_alpha = api.expert_combine_backward(g["y"], y_rows, m["alpha"], plan)
        got[f"alpha{i}"] = d_alpha

        def back(d, w, e):
            lo = offsets[e]
            r = rows[lo:lo + d.shape[0]].float()
            a = torch.relu(r @ w["w1"][e].float().T)
            da = (d.float() @ w["w2"][e].float()) * (a > 0)
            got[f"w1 {i} {e}"], got[f"w2 {i} {e}"] = da.T @ r, d.float().T @ a.to(BF16).float()
            return (da @ w["w1"][e].float()).to(BF16)
        d_x = api.expert_rows_backward(experts(d_rows, offsets, L[i], back), plan)
    g = api.block_norm_backward(m["hidden"], None, d_h, d_x, w_before=L[0]["w_before"], eps=EPS)
    return {**got, "w_before0": g["w_before"], "hidden": g["h"]}


def exact(m):
    """The same in 64 bits, by autograd."""
    d = {k: v.double().requires_grad_() for k, v in dict(
        hidden=m["hidden"], head=m["head"], **{"w_before2": m["final"]}).items()}
    for i, w in enumerate(m["layers"]):
        d[f"alpha{i}"] = m["alpha"].double().requires_grad_()
        for n in ("w_after", "gate", "w_before"):
            d[f"{n}{i}"] = w[n].double().requires_grad_()
        for e in range(E):
            for n in ("w1", "w2"):
                d[f"{n} {i} {e}"] = w[n][e].double().requires_grad_()

    def norm(v, w):
        return v * torch.rsqrt(v.square().mean(1, keepdim=True) + EPS) * w
    h = d["hidden"]
    for i in range(len(m["layers"])):
        x = norm(h, d[f"w_before{i}"])
        y = torch.zeros_like(h)
        for e in range(E):
            t, j = torch.nonzero(m["ids"] == e, as_tuple=True)
            o = torch.relu(x[t] @ d[f"w1 {i} {e}"].T) @ d[f"w2 {i} {e}"].T
            y = y.index_add(0, t, o * d[f"alpha{i}"][t, j][:, None])
        h = h + 0.7 * d[f"gate{i}"] * norm(y, d[f"w_after{i}"])
    live = torch.nonzero(m["targets"] >= 0)[:, 0]
    logp = torch.log_softmax(norm(h, d["w_before2"])[live] @ d["head"].T, 1)
    loss = -logp[torch.arange(live.numel()), m["targets"][live].long()].mean()
    return dict(loss=loss.detach(), **dict(zip(d, torch.autograd.grad(loss, list(d.values())))))


def compare(got, ref):
    assert set(got) == set(ref)
    assert abs(float(got["loss"] / ref["loss"]) - 1) <= 2.0 ** -8
    for name, r in ref.items():
        if name.startswith("alpha"):
            r = torch.where(got[name] == 0, 0.0, r)  # unused slots have no gradient
        size = r.norm()
        rel = float((got[name].double() - r).norm() / size) if size > 0 else 0.0
        behind = name in ("head", "w_before2", "w_after1", "gate1", "alpha1")
        assert rel <= (SMOOTH if behind or name.startswith("w2 1") else THROUGH_RELU), (name, rel)


def test_step():
    m = make(1)
    compare(step(m), exact(m))


def test_steps_are_the_same_bits():
    m = make(2)
    a, b = step(m), step(m)
    assert all(torch.equal(a[k], b[k]) for k in a)


def test_a_captured_step():
    """The calls of a step in a graph, while an eager step of the same tensors is kept."""
    m = make(3)
    plan = api.expert_plan(m["ids"], E=E)
    h, w = m["hidden"], m["layers"][0]
    opt = dict(w_after=w["w_after"], gate=w["gate"], w_before=w["w_before"], eps=EPS)
    grad = torch.full((T,), 1 / T, device="cuda")

    def run():
        p = api.expert_plan(m["ids"], E=E)
        rows = api.expert_rows(h, p)
        y = api.expert_combine(rows, m["alpha"], p)
        o, x = api.block_norm(h, y, **opt)
        loss, lse = api.head_loss(x, m["head"], m["targets"])
        d_x, d_head = api.head_loss_backward(x, m["head"], m["targets"], lse, grad)
        g = api.block_norm_backward(h, y, None, d_x, **opt)
        d_rows, d_alpha = api.expert_combine_backward(g["y"], rows, m["alpha"], p)
        n = plan.offsets[E:]
        return [o, x, loss, lse, d_x, d_head, *g.values(), d_alpha,
                api.expert_rows_backward(d_rows, p), n]
    want = run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for t in got[:-1]:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
