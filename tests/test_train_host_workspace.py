"""The workspace of a head's loss holds what its kernels leave there (no GPU needed): of
up to 64 rows every CTA, one for each row of W where there are few, leaves a maximum and
a sum for 32 or 64 columns, behind the packed rows."""
import shutil
from pathlib import Path

import pytest

pytestmark = pytest.mark.skipif(shutil.which("nvcc") is None and
                                not Path("/usr/local/cuda/bin/nvcc").exists(),
                                reason="needs nvcc to build the library")


@pytest.mark.parametrize("rows,columns", [(1, 32), (32, 32), (33, 64), (64, 64)])
@pytest.mark.parametrize("vocab", [1, 8, 9, 17, 100, 140, 1000, 2000, 4500, 5000, 70000])
def test_sums_of_few_rows(rows, columns, vocab):
    from paper_2608_01784_gb300 import build, _binding as B
    build.build()
    B.load()
    ctas = min(vocab, 100)  # (with 148 or 152 SMs rows of W are shared out to as many or more)
    for k in (1, 64, 2048):
        packed = 64 * (-(-k // 8) * 8) * 2
        assert B.reflex_head_loss_workspace_size(rows, vocab, k) >= packed + ctas * columns * 8
