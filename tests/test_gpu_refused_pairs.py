"""A pair that a layer leaves out (an expert that does not exist) counts nothing,
whatever its weight is."""
import pytest
import torch

from paper_2608_01784_gb300 import _binding as B
from paper_2608_01784_gb300 import api
from tests.test_gpu_fp8 import BF16, experts_layer, normal, routing

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [128, 192, 256, 2048, 2112])
@pytest.mark.parametrize("T", [5, 200])
@pytest.mark.parametrize("weight", [float("nan"), float("inf"), -float("inf")])
def test_a_refused_pair_counts_nothing(d, T, weight):
    E, inter, k_max = 6, 64, 4
    w = experts_layer(d, d, E, inter)
    h = normal(1, T, d, dtype=BF16)
    ids, alpha, k = routing(1, T, E, k_max, lo=3)
    op = api.ExpertsFp8(w, d=d, E=E, inter=inter, k_max=k_max, max_tokens=T)
    bad = ids.clone()
    bad[3, 1], bad[4, 0] = E, -5
    none = alpha.clone()
    none[3, 1] = none[4, 0] = 0.0
    want = op.forward(h, bad, none, k, residual=True)
    assert op.status() == B.REFLEX_EINVAL
    odd = none.clone()
    odd[3, 1] = odd[4, 0] = weight
    out = op.forward(h, bad, odd, k, residual=True)
    assert op.status() == B.REFLEX_EINVAL
    assert torch.equal(out, want) and bool(out.isfinite().all())


def test_counts_past_the_experts():
    """Slots that a clamped count leaves out, with weights of any value."""
    d, E, inter, k_max, T = 256, 2, 64, 4, 200
    w = experts_layer(3, d, E, inter)
    h = normal(1, T, d, dtype=BF16)
    ids, alpha, k = routing(1, T, E, k_max, lo=2)
    op = api.ExpertsFp8(w, d=d, E=E, inter=inter, k_max=k_max, max_tokens=T)
    want = op.forward(h, ids, alpha, k)
    assert op.status() == B.REFLEX_OK
    alpha[:, E:] = float("nan")
    out = op.forward(h, ids, alpha, torch.full_like(k, k_max))
    assert op.status() == B.REFLEX_EKRANGE and torch.equal(out, want)
