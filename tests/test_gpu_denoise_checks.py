"""Tensors that the first kernels of a forward could not read are refused before them."""
import pytest
import torch

from paper_2608_01784_gb300 import _binding as B
from paper_2608_01784_gb300 import denoise
from tests.test_gpu_denoise import CFG, buffers, net, start  # noqa: F401

pytestmark = pytest.mark.gpu


def params():
    return B.make_params(**CFG.alloc_params())


def test_hidden_states_of_another_type(net):  # noqa: F811
    """Refused before the first kernel: the counts stay as they were."""
    state, nb, hidden, u = start(0)
    tokens, conf = buffers()
    net.k.fill_(-7)
    with pytest.raises(ValueError):
        net.forward(state, params(), hidden.float(), u, tokens, conf, nb, 0.5)
    assert bool((net.k == -7).all())


def test_routers_of_another_shape(net):  # noqa: F811
    head = net.head.codes, net.head.scales
    shape = dict(d=CFG.d, E=CFG.E, inter=CFG.inter, k_max=CFG.k_max, max_tokens=8)
    w = net.layers[0]["w_router"]
    for bad in (w[:, :128].contiguous(), w[:4], w.float(), w.t().contiguous().t(), w.cpu()):
        for layers in ([dict(net.layers[0], w_router=bad)],
                       [net.layers[1], dict(net.layers[0], w_router=bad)]):
            with pytest.raises(ValueError):
                denoise.DenoiserFp8(layers, head, **shape)
