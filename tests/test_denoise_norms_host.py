"""A layer's norms that a denoiser refuses (no GPU needed)."""
import pytest
import torch

from paper_2608_01784_gb300.denoise import _norms


@pytest.mark.parametrize("norms", [{}, dict(w_after=torch.ones(8)), dict(scale=0.5),
                                   dict(w_before=None), dict(w_before=torch.ones(8)),
                                   dict(w_before=torch.ones(8), w_behind=torch.ones(8))])
def test_refused(norms):
    layer = dict(w_router=torch.zeros(4, 8), norms=norms)
    with pytest.raises(ValueError):
        _norms([layer], 8, None)
    with pytest.raises(ValueError):
        _norms([layer, dict(w_router=torch.zeros(4, 8))], 8, None)


def test_none():
    assert _norms([dict(w_router=torch.zeros(4, 8))], 8, None) is None
    with pytest.raises(ValueError):
        _norms([dict(w_router=torch.zeros(4, 8))], 8, torch.ones(8))
