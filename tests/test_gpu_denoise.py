"""Whole denoising forwards in 8 bits: the steps together give what they give one
by one, eagerly and in a replayed graph, and a generation ends with every position
committed."""
import pytest
import torch

from paper_2608_01784_gb300 import _binding as B
from paper_2608_01784_gb300 import api, denoise, trajectory
from paper_2608_01784_gb300 import workloads as W

pytestmark = pytest.mark.gpu
CFG = W.CONFIGS["tiny_fp32"].with_(dtype="bf16", n_seq=2)
VOCAB = 777


def draw(g, *shape):
    return (torch.randn(*shape, generator=g, device="cuda") * shape[-1] ** -0.5).bfloat16()


@pytest.fixture(scope="module")
def net():
    g = torch.Generator(device="cuda").manual_seed(1)
    layers = [denoise.quantize_layer(draw(g, CFG.E, CFG.d), draw(g, CFG.E, 2 * CFG.inter, CFG.d),
                                     draw(g, CFG.E, CFG.d, CFG.inter)) for _ in range(3)]
    return denoise.DenoiserFp8(layers, api.quantize_fp8(draw(g, VOCAB, CFG.d), 128), d=CFG.d,
                               E=CFG.E, inter=CFG.inter, k_max=CFG.k_max, max_tokens=CFG.T + 5)


def start(seed):
    st = trajectory.initial_state(W.make_state(CFG, seed))
    nb = torch.from_numpy(trajectory.num_blocks(st)).cuda()
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (api.state_to_device(st), nb, draw(g, CFG.T, CFG.d) * 16,
            torch.rand(CFG.T, generator=g, device="cuda"))


def buffers():
    return (torch.empty(CFG.T, dtype=torch.int32, device="cuda"),
            torch.empty(CFG.T, device="cuda"))


def one_by_one(net, state, nb, hidden, u, theta):
    """The same forward from the operators' own entry points."""
    params = B.make_params(**CFG.alloc_params())
    k, _, _ = api.allocate(state, params, CFG.E)
    h = hidden
    for w in net.layers:
        ids = torch.empty(CFG.T, CFG.k_max, dtype=torch.int32, device="cuda")
        alpha = torch.empty(CFG.T, CFG.k_max, device="cuda")
        assert B.reflex_route_noalloc(B.REFLEX_DTYPE_BF16, h, w["w_router"], k, CFG.T, CFG.d,
                                      CFG.E, CFG.k_max, B.REFLEX_FLAG_RENORM_TOPK, ids,
                                      alpha) == B.REFLEX_OK
        layer = api.ExpertsFp8(w, d=CFG.d, E=CFG.E, inter=CFG.inter, k_max=CFG.k_max,
                               max_tokens=CFG.T)
        h = layer.forward(h, ids, alpha, k, residual=True)
    head = api.LinearFp8(net.head.codes, net.head.scales, max_rows=CFG.T)
    tokens, conf = api.sample(head.forward(h), u, masked=state["masked"])
    api.update_state(state, conf, nb, theta)
    return tokens, conf


@pytest.mark.parametrize("seed", [0, 3])
def test_forward_is_its_steps(net, seed):
    state, nb, hidden, u = start(seed)
    want, _, _, _ = start(seed)
    tokens, conf = buffers()
    for step in range(3):
        t0, c0 = one_by_one(net, want, nb, hidden, u, 0.05)
        net.forward(state, B.make_params(**CFG.alloc_params()), hidden, u, tokens, conf, nb, 0.05)
        assert net.status() == B.REFLEX_OK
        assert torch.equal(tokens, t0) and torch.equal(conf, c0)
        for name, t in want.items():
            assert torch.equal(state[name], t), name
        u = torch.rand(CFG.T, generator=torch.Generator(device="cuda").manual_seed(step),
                       device="cuda")


def test_replayed_graph_is_the_eager_forward(net):
    params = B.make_params(**CFG.alloc_params())
    eager, nb, hidden, u = start(5)
    state, _, _, _ = start(5)
    tokens, conf = buffers()
    t0, c0 = buffers()
    committed = torch.empty(2, dtype=torch.int32, device="cuda")
    net.forward(eager, params, hidden, u, t0, c0, nb, 0.05)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, capture_error_mode="relaxed"):
        net.forward(state, params, hidden, u, tokens, conf, nb, 0.05, committed=committed)
    for _ in range(2):
        graph.replay()
        assert torch.equal(tokens, t0) and torch.equal(conf, c0)
        for name, t in eager.items():
            assert torch.equal(state[name], t), name
        net.forward(eager, params, hidden, u, t0, c0, nb, 0.05)


def test_generation_ends():
    done = denoise.main(2)
    target = done["state"]["block_id"] > 0
    assert not bool(done["state"]["masked"].any())
    assert bool(((done["text"] >= 0) == target).all())
    assert bool((done["text"] < done["vocab"]).all())
    assert 2 <= done["forwards"] <= int(target.sum())


def test_refusals(net):
    state, nb, hidden, u = start(0)
    tokens, conf = buffers()
    params = B.make_params(**CFG.alloc_params())
    with pytest.raises(ValueError):
        denoise.DenoiserFp8([], (net.head.codes, net.head.scales), d=CFG.d, E=CFG.E,
                            inter=CFG.inter, k_max=CFG.k_max, max_tokens=8)
    with pytest.raises(ValueError):
        net.forward(state, params, torch.cat([hidden, hidden]), u, tokens, conf, nb, 0.5)
    with pytest.raises(ValueError):
        net.forward(state, params, hidden, u[:-1], tokens, conf, nb, 0.5)
    narrow = api.quantize_fp8(torch.ones(16, 128, device="cuda"), 128)
    with pytest.raises(ValueError):
        denoise.DenoiserFp8(net.layers, narrow, d=CFG.d, E=CFG.E, inter=CFG.inter,
                            k_max=CFG.k_max, max_tokens=8)
