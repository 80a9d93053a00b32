"""Rows too wide for the sums and copies of pair rows are refused (no GPU needed)."""
import shutil
from pathlib import Path

import pytest

from test_train_host import COMBINE, COMBINE_GRAD, ROWS, call

pytestmark = pytest.mark.skipif(shutil.which("nvcc") is None and
                                not Path("/usr/local/cuda/bin/nvcc").exists(),
                                reason="needs nvcc to build the library")


@pytest.mark.parametrize("d", [(1 << 30) + 1, (1 << 31) - 1])
@pytest.mark.parametrize("dtype", [0, 1])
def test_wide_rows(d, dtype):
    from paper_2608_01784_gb300 import build, _binding as B
    build.build()
    B.load()
    for fn, good in ((B.reflex_expert_rows, ROWS), (B.reflex_expert_combine, COMBINE),
                     (B.reflex_expert_combine_backward, COMBINE_GRAD)):
        wide = {n: d for n in good if n == "d" or n.startswith("ld")}
        assert call(fn, good, dtype=dtype, **wide) == B.REFLEX_EUNSUPPORTED
        assert call(fn, good, dtype=dtype, **wide, T=0) == B.REFLEX_OK
