"""A whole forward takes no memory from the allocator, with and without a place for
its commits."""
import pytest
import torch

from paper_2608_01784_gb300 import _binding as B
from tests.test_gpu_denoise import CFG, buffers, net, start  # noqa: F401

pytestmark = pytest.mark.gpu


def params():
    return B.make_params(**CFG.alloc_params())


def test_a_forward_allocates_nothing(net):  # noqa: F811
    state, nb, hidden, u = start(1)
    tokens, conf = buffers()
    for _ in range(2):
        before = torch.cuda.memory_stats()["allocation.all.allocated"]
        committed = net.forward(state, params(), hidden, u, tokens, conf, nb, 0.5)
        assert torch.cuda.memory_stats()["allocation.all.allocated"] == before
    assert committed.shape == (2,) and committed.dtype == torch.int32
    assert int(committed.sum()) > 0
    own = torch.zeros(2, dtype=torch.int32, device="cuda")
    assert net.forward(state, params(), hidden, u, tokens, conf, nb, 0.5, committed=own) is own
