"""Nothing is rounded between the products of a few pairs and their weighted sum: on
whole numbers, of which every code, product and sum is exact, the layer is too."""
import pytest
import torch

from paper_2608_01784_gb300 import _binding as B
from paper_2608_01784_gb300 import api
from tests.test_gpu_fp8 import BF16, experts64

pytestmark = pytest.mark.gpu


def whole_number_layer(d, inter):
    """Two experts whose outputs, some thousands, differ by less than 256, so that the
    difference fits bf16.  Each block holds a 448 (14 * 32) and so has a power of two
    for a scale; gates are 32, where silu(g) = g."""
    g = torch.Generator().manual_seed(inter)
    small = lambda *s: torch.randint(1, 15, s, generator=g).float()  # noqa: E731
    hidden = torch.zeros(d)
    hidden[0], hidden[1] = 256.0, 448.0
    gate, up = torch.zeros(inter, d), torch.zeros(inter, d)
    gate[:, 0], gate[::128, 2] = 256.0, 448.0
    up[:, 0] = small(inter) * 32
    up[::128, 0] = 448.0
    down = small(d, inter) * 32
    down[::128, ::128] = 448.0
    other = down.clone()
    at = torch.arange(d)
    other[at, 1 + at % 50] = 480.0 - down[at, 1 + at % 50]  # m becomes 15 - m
    gate_up = torch.cat([gate * 2.0 ** -11, up * 2.0 ** -13])
    return hidden, torch.stack([gate_up, gate_up]), torch.stack([down, other]) * 2.0 ** -10


@pytest.mark.parametrize("T", [1, 5])
@pytest.mark.parametrize("inter", [128, 256])
def test_pair_outputs_are_not_rounded(T, inter):
    d, k_max = 256, 2
    hidden, gate_up, down = whole_number_layer(d, inter)
    w = api.quantize_experts(gate_up.cuda(), down.cuda())
    h = hidden.to(BF16).cuda().repeat(T, 1)
    ids = torch.tensor([[0, 1]], dtype=torch.int32, device="cuda").repeat(T, 1)
    alpha = torch.tensor([[1.0, -1.0]], device="cuda").repeat(T, 1)
    k = torch.full((T,), 2, dtype=torch.int32, device="cuda")
    op = api.ExpertsFp8(w, d=d, E=2, inter=inter, k_max=k_max, max_tokens=T)
    out = op.forward(h, ids, alpha, k)
    assert op.status() == B.REFLEX_OK
    ref = experts64(h, ids, alpha, w, inter)
    assert torch.equal(ref, ref.to(BF16).double()) and bool((ref != 0).all())
    assert torch.equal(out.double(), ref)
