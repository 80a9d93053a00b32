"""Sizes of zero come back from the entry points around the experts like any other (no
GPU needed)."""
import shutil
from pathlib import Path

import pytest

from test_train_host import COMBINE, COMBINE_GRAD, HEAD, HEAD_GRAD, NORM, PLAN, ROWS, call

pytestmark = pytest.mark.skipif(shutil.which("nvcc") is None and
                                not Path("/usr/local/cuda/bin/nvcc").exists(),
                                reason="needs nvcc to build the library")


@pytest.fixture(scope="module")
def B():
    from paper_2608_01784_gb300 import build, _binding
    build.build()
    _binding.load()
    return _binding


@pytest.mark.parametrize("vocab,k", [(1, 1), (600, 60), (1 << 24, 64)])
def test_head_of_no_rows(B, vocab, k):
    sizes = dict(rows=0, vocab=vocab, k=k)
    for fn, good, size in ((B.reflex_head_loss, HEAD, B.reflex_head_loss_workspace_size),
                           (B.reflex_head_loss_backward, HEAD_GRAD,
                            B.reflex_head_loss_backward_workspace_size)):
        need = size(0, vocab, k)
        assert 0 < need <= size(1, vocab, k)
        wide = {n: k + 8 - k % 8 for n in ("ld_hidden", "ldw", "ld_d_hidden", "ld_d_w") if n in good}
        assert call(fn, good, **sizes, **wide, ws_bytes=need - 1) == B.REFLEX_EWORKSPACE


def test_nothing_to_do(B):
    assert B.reflex_block_norm_workspace_size(0, 100) > 0
    assert B.reflex_expert_plan_workspace_size(0, 8, 4) > 0
    assert call(B.reflex_block_norm, NORM, rows=0) == B.REFLEX_OK
    assert call(B.reflex_expert_plan, PLAN, T=0, ws_bytes=0) == B.REFLEX_EWORKSPACE
    for fn, good in ((B.reflex_expert_rows, ROWS), (B.reflex_expert_combine, COMBINE),
                     (B.reflex_expert_combine_backward, COMBINE_GRAD)):
        assert call(fn, good, T=0) == B.REFLEX_OK
    assert call(B.reflex_expert_rows, ROWS, cap_rows=0) == B.REFLEX_OK
