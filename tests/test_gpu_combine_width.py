"""The weighted sum of Eq. 2 at widths that are no multiple of 256, with more
slots than the last columns of a row have lanes: every slot counts in every
column."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,k_max", [(64, 12), (192, 32), (320, 12), (448, 16), (2112, 12)])
def test_every_slot_in_every_column(d, k_max):
    import torch
    from paper_2608_01784_gb300 import _binding as B
    from paper_2608_01784_gb300 import api
    T, E, inter = 37, 40, 64
    g = torch.Generator().manual_seed(d)
    w = {n: (torch.randn(*s, generator=g) * 0.1).cuda() for n, s in (
        ("w_router", (E, d)), ("w_gate_up", (E, 2 * inter, d)), ("w_down", (E, d, inter)))}
    h = torch.randn(T, d, generator=g).cuda()
    k = (torch.arange(T, dtype=torch.int32) % k_max + 1).cuda()
    moe = api.MoELayer(w, dtype="f32", d=d, E=E, inter=inter, shared_inter=0, k_max=k_max,
                       max_tokens=T)
    out = moe.forward(h, k)
    assert moe.status() == B.REFLEX_OK
    rec = moe.record()
    ids, alpha = rec["ids"].long(), rec["alpha"].double()
    gate, up = w["w_gate_up"].double().split(inter, 1)
    x = h.double()
    a = torch.einsum("td,eid->tei", x, gate)
    a = a * torch.sigmoid(a) * torch.einsum("td,eid->tei", x, up)
    y = torch.einsum("tei,edi->ted", a, w["w_down"].double())
    pick = y.gather(1, ids.clamp(min=0)[..., None].expand(-1, -1, d))
    ref = torch.where((ids >= 0)[..., None], pick * alpha[..., None], 0.0).sum(1)
    # fp32 sums of d, inter and k_max terms, the project's bound for fp32 layers
    assert float((out.double() - ref).norm() / ref.norm()) <= 1e-5
    assert np.isfinite(float(out.sum()))
