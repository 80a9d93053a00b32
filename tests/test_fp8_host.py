"""Host-side refusals of the 8-bit products and of sampling (no GPU needed): every
call here returns its status before anything is enqueued."""
import shutil
from pathlib import Path

import pytest

pytestmark = pytest.mark.skipif(shutil.which("nvcc") is None and
                                not Path("/usr/local/cuda/bin/nvcc").exists(),
                                reason="needs nvcc to build the library")
P = 1 << 20  # an address that no call gets as far as reading
BIG = 1 << 31


@pytest.fixture(scope="module")
def B():
    from paper_2608_01784_gb300 import build, _binding
    build.build()
    _binding.load()
    return _binding


def call(fn, good, **changes):
    return fn(*{**good, **changes}.values(), stream=0, check=False)


QUANTIZE = dict(dtype=1, x=P, rows=4, cols=200, ldx=200, block_rows=1, codes=P, ldc=200, scales=P,
                lds=2)


@pytest.mark.parametrize("changes", [
    dict(dtype=2), dict(rows=-1), dict(cols=-1), dict(block_rows=64), dict(block_rows=0),
    dict(x=None), dict(codes=None), dict(scales=None), dict(ldx=199), dict(ldc=199), dict(lds=1),
    dict(x=P + 1), dict(dtype=0, x=P + 2), dict(scales=P + 2)])
def test_quantize_refuses(B, changes):
    assert call(B.reflex_quantize_fp8, QUANTIZE, **changes) == B.REFLEX_EINVAL


@pytest.mark.parametrize("changes", [dict(rows=0), dict(cols=0), dict(rows=0, x=None)])
def test_quantize_of_nothing(B, changes):
    assert call(B.reflex_quantize_fp8, QUANTIZE, **changes) == B.REFLEX_OK


def test_quantize_of_too_much(B):
    wide = dict(cols=BIG, ldx=BIG, ldc=BIG, lds=BIG)
    assert call(B.reflex_quantize_fp8, QUANTIZE, **wide) == B.REFLEX_EUNSUPPORTED


MATMUL = dict(a=P, lda=208, a_scales=P, ldas=2, b=P, ldb=208, b_scales=P, ldbs=2, M=4, N=10, K=200,
              out_dtype=1, out=P, ldo=10, dev_status=None)
PRODUCT = [dict(M=-1), dict(N=0), dict(K=0), dict(out_dtype=2), dict(ldo=9), dict(out=None),
           dict(out=P + 1), dict(out_dtype=0, out=P + 2)]


@pytest.mark.parametrize("changes", PRODUCT + [
    dict(a=None), dict(b=None), dict(a_scales=None), dict(b_scales=None), dict(lda=200),
    dict(lda=192), dict(ldb=200), dict(ldb=192), dict(ldas=1), dict(ldbs=1), dict(a=P + 8),
    dict(b=P + 8), dict(a_scales=P + 2), dict(b_scales=P + 2)])
def test_matmul_refuses(B, changes):
    # (with an error word: a refused call must not touch it)
    assert call(B.reflex_matmul_fp8, MATMUL, dev_status=P, **changes) == B.REFLEX_EINVAL


def test_matmul_of_nothing_and_of_too_much(B):
    assert call(B.reflex_matmul_fp8, MATMUL, M=0, a=None, a_scales=None) == B.REFLEX_OK
    huge = (1 << 30) + 1
    assert call(B.reflex_matmul_fp8, MATMUL, M=huge) == B.REFLEX_EUNSUPPORTED
    assert call(B.reflex_matmul_fp8, MATMUL, N=huge, ldo=huge) == B.REFLEX_EUNSUPPORTED
    assert call(B.reflex_matmul_fp8, MATMUL, M=1 << 30, N=1 << 30,
                ldo=1 << 30) == B.REFLEX_EUNSUPPORTED


LINEAR = dict(dtype=1, x=P, ldx=200, w=P, ldw=208, w_scales=P, ldws=2, M=4, N=10, K=200,
              out_dtype=1, out=P, ldo=10, workspace=P, ws_bytes=P)


@pytest.mark.parametrize("changes", PRODUCT + [
    dict(dtype=2), dict(x=None), dict(w=None), dict(w_scales=None), dict(ldx=199), dict(ldw=200),
    dict(ldws=1), dict(x=P + 1), dict(dtype=0, x=P + 2), dict(w=P + 8), dict(w_scales=P + 2)])
def test_linear_refuses(B, changes):
    assert call(B.reflex_linear_fp8, LINEAR, **changes) == B.REFLEX_EINVAL


def test_linear_workspace(B):
    size = B.reflex_linear_fp8_workspace_size
    assert size(-1, 200) == 0 and size(4, 0) == 0
    assert 0 < size(0, 200) < size(4, 200) < size(4, 20000) < size(400, 20000)
    for changes in (dict(workspace=None), dict(workspace=P + 64),
                    dict(ws_bytes=size(4, 200) - 1)):
        assert call(B.reflex_linear_fp8, LINEAR, **changes) == B.REFLEX_EWORKSPACE


EXPERTS = dict(hidden=P, ids=P, alpha=P, k=P, w_gate_up=P, gate_up_scales=P, w_down=P,
               down_scales=P, T=4, d=128, E=8, inter=64, k_max=4, flags=0, workspace=P,
               ws_bytes=P, out=P)


@pytest.mark.parametrize("changes", [
    dict(T=-1), dict(d=100), dict(d=0), dict(E=0), dict(E=1025), dict(inter=65), dict(inter=0),
    dict(k_max=0), dict(k_max=33), dict(T=1 << 28, k_max=32), dict(flags=4096)] +
    [{name: None} for name in ("hidden", "ids", "alpha", "k", "w_gate_up", "gate_up_scales",
                               "w_down", "down_scales", "out")] +
    [{name: P + 8} for name in ("hidden", "w_gate_up", "w_down", "out")] +
    [{name: P + 2} for name in ("ids", "alpha", "k", "gate_up_scales", "down_scales")])
def test_experts_refuse(B, changes):
    assert call(B.reflex_experts_fp8, EXPERTS, **changes) == B.REFLEX_EINVAL


def test_experts_workspace(B):
    size = B.reflex_experts_fp8_workspace_size
    assert size(4, 128, 8, 64, 33) == 0 and size(4, 100, 8, 64, 4) == 0
    assert 0 < size(0, 128, 8, 64, 4) < size(4, 128, 8, 64, 4) < size(4096, 128, 8, 64, 4)
    need = size(4, 128, 8, 64, 4)
    for changes in (dict(workspace=None), dict(workspace=P + 64), dict(ws_bytes=need - 1)):
        assert call(B.reflex_experts_fp8, EXPERTS, **changes) == B.REFLEX_EWORKSPACE


SAMPLE = dict(dtype=1, logits=P, ld=100, rows=4, vocab=100, temperature=None, top_k=None,
              top_p=None, min_p=None, u=P, masked=None, tokens_out=P, conf_out=P,
              dev_status=None)


@pytest.mark.parametrize("changes", [
    dict(dtype=2), dict(rows=-1), dict(vocab=0), dict(ld=99), dict(logits=None), dict(u=None),
    dict(tokens_out=None), dict(conf_out=None), dict(logits=P + 1), dict(dtype=0, logits=P + 2)])
def test_sample_refuses(B, changes):
    assert call(B.reflex_sample, SAMPLE, **changes) == B.REFLEX_EINVAL


def test_sample_of_nothing_and_of_too_much(B):
    assert call(B.reflex_sample, SAMPLE, rows=0, logits=None) == B.REFLEX_OK
    wide = (1 << 18) + 1
    assert call(B.reflex_sample, SAMPLE, vocab=wide, ld=wide) == B.REFLEX_EUNSUPPORTED
    assert call(B.reflex_sample, SAMPLE, rows=(1 << 27) + 1) == B.REFLEX_EUNSUPPORTED
