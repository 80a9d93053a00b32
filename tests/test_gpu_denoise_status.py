"""An error that one layer of a forward meets is reported, whatever the later ones do."""
import pytest

from paper_2608_01784_gb300 import _binding as B
from tests.test_gpu_denoise import CFG, buffers, net, start  # noqa: F401

pytestmark = pytest.mark.gpu


def params():
    return B.make_params(**CFG.alloc_params())


@pytest.mark.parametrize("layer", [0, 1, 2])
def test_an_error_of_any_layer_is_kept(net, layer, monkeypatch):  # noqa: F811
    state, nb, hidden, u = start(0)
    tokens, conf = buffers()
    plain, calls = net.experts.forward, []

    def forward(h, ids, *args, **kw):
        calls.append(0)
        if len(calls) == layer + 1:
            ids = ids.clone()
            ids[2, 0] = CFG.E
        return plain(h, ids, *args, **kw)
    monkeypatch.setattr(net.experts, "forward", forward)
    net.forward(state, params(), hidden, u, tokens, conf, nb, 0.5)
    assert net.status() == B.REFLEX_EINVAL
    monkeypatch.undo()
    net.forward(state, params(), hidden, u, tokens, conf, nb, 0.5)
    assert net.status() == B.REFLEX_OK


@pytest.mark.parametrize("layer", [1, 2])
def test_an_error_of_any_router_is_kept(net, layer, monkeypatch):  # noqa: F811
    state, nb, hidden, u = start(0)
    tokens, conf = buffers()
    plain, calls = net.router.forward, []

    def forward(h, k, *args, **kw):
        calls.append(0)
        if len(calls) == layer:
            k = k.clone()
            k[5] = CFG.k_max + 9
        return plain(h, k, *args, **kw)
    monkeypatch.setattr(net.router, "forward", forward)
    net.forward(state, params(), hidden, u, tokens, conf, nb, 0.5)
    assert net.status() == B.REFLEX_EKRANGE
    monkeypatch.undo()
    net.forward(state, params(), hidden, u, tokens, conf, nb, 0.5)
    assert net.status() == B.REFLEX_OK
