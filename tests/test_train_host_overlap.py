"""A gradient of the head's weights that would be written over the weights it reads is
refused, wherever it starts (no GPU needed: refused before anything is enqueued)."""
import shutil
from pathlib import Path

import pytest
import torch

pytestmark = pytest.mark.skipif(shutil.which("nvcc") is None and
                                not Path("/usr/local/cuda/bin/nvcc").exists(),
                                reason="needs nvcc to build the library")
P, LD, VOCAB, K = 1 << 20, 104, 50, 100
END = P + 2 * ((VOCAB - 1) * LD + K)  # behind the weights


@pytest.fixture(scope="module")
def B():
    from paper_2608_01784_gb300 import build, _binding
    build.build()
    _binding.load()
    return _binding


def refused(B, **changes):
    args = dict(hidden=1 << 30, ld_hidden=K, w=P, ldw=LD, targets=1 << 30, lse=1 << 30, grad=1 << 30,
                rows=4, vocab=VOCAB, k=K, d_hidden_dtype=1, d_hidden=1 << 31, ld_d_hidden=K,
                d_w_dtype=1, d_w=P, ld_d_w=LD, dev_status=None, workspace=1 << 32, ws_bytes=1 << 40)
    assert set(changes) <= set(args)
    return B.reflex_head_loss_backward(*{**args, **changes}.values(), stream=0, check=False)


@pytest.mark.parametrize("changes", [
    dict(), dict(d_w=P + 2 * LD), dict(d_w=P - 2 * LD), dict(d_w=P + 2), dict(d_w=P + 2 * K - 2),
    dict(d_w=END - 2), dict(d_w=P - 2 * ((VOCAB - 1) * LD + K) + 2), dict(d_w=P + 2, ld_d_w=LD + 1),
    dict(d_w_dtype=0), dict(d_w_dtype=0, d_w=END - 4), dict(d_w_dtype=0, d_w=P - 4, ld_d_w=K),
    dict(rows=0)])
def test_refused(B, changes):
    assert refused(B, **changes) == B.REFLEX_EINVAL


@pytest.mark.parametrize("changes", [
    dict(d_hidden=P), dict(d_hidden=END - 2), dict(d_hidden=P - 2 * (3 * K + K) + 2),
    dict(d_hidden=P + 8, d_hidden_dtype=0, d_w=None), dict(d_hidden=(1 << 28) + 2 * LD, d_w=1 << 28),
    dict(d_hidden=(1 << 28) - 2 * 3 * K, d_w=1 << 28)])
def test_gradients_of_the_rows_refused(B, changes):
    assert refused(B, **{**dict(d_w=1 << 29), **changes}) == B.REFLEX_EINVAL


def test_matrices_in_one_buffer():
    """Halves of wider rows and neighbours share nothing."""
    from paper_2608_01784_gb300.train import _overlap
    wide = torch.zeros(2 * VOCAB, 2 * LD, dtype=torch.bfloat16)
    left, right = wide[:VOCAB, :K], wide[:VOCAB, LD:LD + K]
    below = wide[VOCAB:, :K]

    def shared(a, b):
        got = _overlap(a, a.stride(0), b, b.stride(0))
        assert got == _overlap(b, b.stride(0), a, a.stride(0))
        return got
    assert not shared(left, right) and not shared(left, below) and not shared(right, below)
    assert shared(left, left) and shared(left, wide[1:VOCAB + 1, :K])
    assert shared(left, wide[:VOCAB, K - 1:2 * K - 1]) and shared(right, wide[:VOCAB, K + 3:2 * K + 3])
    flat = wide.view(-1)
    assert not shared(flat[:VOCAB * K].view(VOCAB, K), flat[VOCAB * K:2 * VOCAB * K].view(VOCAB, K))
    assert shared(flat[:VOCAB * K].view(VOCAB, K), flat[VOCAB * K - 1:2 * VOCAB * K - 1].view(VOCAB, K))
    # another type in the same bytes
    assert shared(flat[:VOCAB * 2 * K].view(torch.float32).view(VOCAB, K), flat[:VOCAB * K].view(VOCAB, K))
