"""Addresses that a kernel could not read or write a 32-bit word at are refused before
anything is enqueued (no GPU needed)."""
import pytest

from tests.test_fp8_host import MATMUL, P, SAMPLE, B, call, pytestmark  # noqa: F401


@pytest.mark.parametrize("name", ["temperature", "top_k", "top_p", "min_p", "u", "tokens_out",
                                  "conf_out", "dev_status"])
@pytest.mark.parametrize("off", [1, 2])
def test_sample_refuses_odd_addresses(B, name, off):  # noqa: F811
    assert call(B.reflex_sample, SAMPLE, **{name: P + off}) == B.REFLEX_EINVAL


@pytest.mark.parametrize("off", [1, 2])
def test_matmul_refuses_odd_error_words(B, off):  # noqa: F811
    assert call(B.reflex_matmul_fp8, MATMUL, dev_status=P + off) == B.REFLEX_EINVAL
    assert call(B.reflex_matmul_fp8, MATMUL, M=0, dev_status=P + off) == B.REFLEX_EINVAL
