"""Error words that a kernel could not write are refused before anything is enqueued."""
import pytest
import torch

from paper_2608_01784_gb300 import _binding as B
from paper_2608_01784_gb300 import api
from tests.test_gpu_fp8 import normal

pytestmark = pytest.mark.gpu


def bad_words():
    return dict(host=torch.zeros(1, dtype=torch.int32),
                empty=torch.zeros(0, dtype=torch.int32, device="cuda"),
                bytes=torch.zeros(1, dtype=torch.uint8, device="cuda"),
                wide=torch.zeros(1, dtype=torch.int64, device="cuda"),
                several=torch.zeros(2, dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("name", ["host", "empty", "bytes", "wide", "several"])
def test_error_words(name, monkeypatch):
    # the entry points themselves are out of reach: a call that is let through fails here
    def enqueued(*args, **kw):
        raise AssertionError("the call went on")
    a, b = api.quantize_fp8(normal(1, 4, 64)), api.quantize_fp8(normal(2, 8, 64), 128)
    z, u = normal(3, 4, 50), torch.full((4,), 0.5, device="cuda")
    monkeypatch.setattr(B, "reflex_matmul_fp8", enqueued)
    monkeypatch.setattr(B, "reflex_sample", enqueued)
    bad = bad_words()[name]
    with pytest.raises(ValueError):
        api.matmul_fp8(*a, *b, status=bad)
    with pytest.raises(ValueError):
        api.sample(z, u, status=bad)


def test_error_words_that_fit():
    a, b = api.quantize_fp8(normal(1, 4, 64)), api.quantize_fp8(normal(2, 8, 64), 128)
    z, u = normal(3, 4, 50), torch.full((4,), 0.5, device="cuda")
    words = torch.full((3,), 77, dtype=torch.int32, device="cuda")
    api.matmul_fp8(*a, *b, status=words[1:2])
    assert words.tolist() == [77, 0, 77]
    words.zero_()
    api.sample(z, u, temperature=torch.full((4,), -1.0, device="cuda"), status=words[2:])
    assert words[:2].tolist() == [0, 0]
    assert B.reflex_read_status(words[2:]) == B.REFLEX_EINVAL
