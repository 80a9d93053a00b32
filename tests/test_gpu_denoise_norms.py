"""Denoising forwards of layers with norms: the steps together give what they give one
by one, in a replayed graph too."""
import pytest
import torch

from paper_2608_01784_gb300 import _binding as B
from paper_2608_01784_gb300 import api, denoise
from tests.test_gpu_denoise import CFG, VOCAB, buffers, draw, start

pytestmark = pytest.mark.gpu


def weight(g):
    return (1 + 0.1 * torch.randn(CFG.d, generator=g, device="cuda")).bfloat16()


def make(final: bool, gates: bool):
    g = torch.Generator(device="cuda").manual_seed(7)
    layers = []
    for i in range(3):
        norms = dict(w_before=weight(g))
        if gates:
            norms.update(w_after=weight(g), gate=draw(g, CFG.d) * 10, scale=0.7)
        layers.append(denoise.quantize_layer(
            draw(g, CFG.E, CFG.d), draw(g, CFG.E, 2 * CFG.inter, CFG.d),
            draw(g, CFG.E, CFG.d, CFG.inter), norms=norms))
    head = api.quantize_fp8(draw(g, VOCAB, CFG.d), 128)
    return layers, head, weight(g) if final else None


def net_of(layers, head, final):
    return denoise.DenoiserFp8(layers, head, d=CFG.d, E=CFG.E, inter=CFG.inter, k_max=CFG.k_max,
                               max_tokens=CFG.T + 3, final_norm=final)


def one_by_one(layers, head, final, state, hidden):
    params = B.make_params(**CFG.alloc_params())
    k, _, _ = api.allocate(state, params, CFG.E)
    stream, x = api.block_norm(hidden, w_before=layers[0]["norms"]["w_before"])
    for i, w in enumerate(layers):
        ids = torch.empty(CFG.T, CFG.k_max, dtype=torch.int32, device="cuda")
        alpha = torch.empty(CFG.T, CFG.k_max, device="cuda")
        assert B.reflex_route_noalloc(B.REFLEX_DTYPE_BF16, x, w["w_router"], k, CFG.T, CFG.d,
                                      CFG.E, CFG.k_max, B.REFLEX_FLAG_RENORM_TOPK, ids,
                                      alpha) == B.REFLEX_OK
        layer = api.ExpertsFp8(w, d=CFG.d, E=CFG.E, inter=CFG.inter, k_max=CFG.k_max,
                               max_tokens=CFG.T)
        y = layer.forward(x, ids, alpha, k)
        n = dict(w["norms"])
        n["w_before"] = layers[i + 1]["norms"]["w_before"] if i + 1 < len(layers) else final
        stream, x = api.block_norm(stream, y, **n)
    return api.LinearFp8(*head, max_rows=CFG.T).forward(stream if final is None else x)


@pytest.mark.parametrize("final,gates", [(True, True), (True, False), (False, True)])
def test_forward_is_its_steps(final, gates):
    layers, head, last = make(final, gates)
    net = net_of(layers, head, last)
    state, nb, hidden, u = start(2)
    params = B.make_params(**CFG.alloc_params())
    want = one_by_one(layers, head, last, state, hidden)
    keep = hidden.clone()
    assert torch.equal(net.logits(state, params, hidden), want)
    assert torch.equal(hidden, keep) and net.status() == B.REFLEX_OK
    assert torch.equal(net.logits(state, params, hidden), want)


def test_replayed_graph_is_the_eager_forward():
    net = net_of(*make(True, True))
    params = B.make_params(**CFG.alloc_params())
    eager, nb, hidden, u = start(5)
    state, _, _, _ = start(5)
    tokens, conf = buffers()
    t0, c0 = buffers()
    net.forward(eager, params, hidden, u, t0, c0, nb, 0.05)
    committed = torch.empty(2, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, capture_error_mode="relaxed"):
        net.forward(state, params, hidden, u, tokens, conf, nb, 0.05, committed=committed)
    graph.replay()
    assert torch.equal(tokens, t0) and torch.equal(conf, c0)
    for name, t in eager.items():
        assert torch.equal(state[name], t), name


def test_refusals():
    layers, head, final = make(True, True)
    plain = dict(layers[0])
    del plain["norms"]
    bad = [([layers[0], plain], None), ([plain], final),
           ([dict(layers[0], norms=dict(w_before=final[:-1]))], None),
           ([dict(layers[0], norms=dict(w_before=final.float()))], None),
           ([dict(layers[0], norms=dict(w_before=final, gate=final.cpu()))], None),
           ([dict(layers[0], norms=dict(w_before=final, other=final))], None),
           (layers, final[:-1])]
    for ls, f in bad:
        with pytest.raises(ValueError):
            net_of(ls, head, f)
