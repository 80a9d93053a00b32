"""Host-side refusals of the calls around the experts (no GPU needed): every call here
returns its status before anything is enqueued."""
import shutil
from pathlib import Path

import pytest

pytestmark = pytest.mark.skipif(shutil.which("nvcc") is None and
                                not Path("/usr/local/cuda/bin/nvcc").exists(),
                                reason="needs nvcc to build the library")
P = 1 << 20  # an address that no call gets as far as reading


@pytest.fixture(scope="module")
def B():
    from paper_2608_01784_gb300 import build, _binding
    build.build()
    _binding.load()
    return _binding


def call(fn, good, **changes):
    return fn(*{**good, **changes}.values(), stream=0, check=False)


STREAM = dict(dtype=1, h=P, ldh=100, y=P, ldy=100, w_after=P, gate=P, ldg=0, w_before=P, scale=1.0,
              eps=1e-6, rows=4, d=100)
NORM = dict(**STREAM, out=P, ldo=100, norm=P, ldn=100)
NORM_GRAD = dict(**STREAM, d_out=P, ld_d_out=100, d_norm=P, ld_d_norm=100, d_h=P, ld_d_h=100,
                 d_y=P, ld_d_y=100, d_gate=P, ld_d_gate=100, d_w_after=P, d_w_before=P,
                 workspace=P, ws_bytes=P << 10)
BAD_STREAM = [dict(dtype=2), dict(h=None), dict(ldh=99), dict(ldy=99), dict(ldg=99), dict(rows=-1),
              dict(d=0), dict(h=P + 1), dict(y=P + 1), dict(gate=P + 1), dict(w_after=P + 1),
              dict(w_before=P + 1), dict(y=None), dict(scale=float("nan")),
              dict(scale=float("inf")), dict(eps=-1.0), dict(eps=float("nan")),
              dict(dtype=0, h=P + 2), dict(dtype=0, w_before=P + 2)]


@pytest.mark.parametrize("changes", BAD_STREAM + [
    dict(out=None, norm=None), dict(w_before=None), dict(ldo=99), dict(ldn=99), dict(out=P + 1),
    dict(norm=P + 1)])
def test_block_norm_refuses(B, changes):
    assert call(B.reflex_block_norm, NORM, **changes) == B.REFLEX_EINVAL


@pytest.mark.parametrize("changes", BAD_STREAM + [
    dict(d_out=None, d_norm=None), dict(d_norm=None), dict(w_before=None), dict(w_after=None),
    dict(gate=None), dict(d_h=None), dict(d_y=None), dict(d_out=P + 1), dict(d_norm=P + 1),
    dict(d_h=P + 1), dict(d_y=P + 1), dict(d_gate=P + 1), dict(d_w_after=P + 1),
    dict(d_w_before=P + 1), dict(ld_d_out=99), dict(ld_d_norm=99), dict(ld_d_h=99),
    dict(ld_d_y=99), dict(ldg=100, ld_d_gate=99)])
def test_block_norm_backward_refuses(B, changes):
    assert call(B.reflex_block_norm_backward, NORM_GRAD, **changes) == B.REFLEX_EINVAL


def test_block_norm_widths_and_workspace(B):
    wide = {n: 16385 for n in ("d", "ldh", "ldy", "ldo", "ldn")}
    assert call(B.reflex_block_norm, NORM, **wide) == B.REFLEX_EUNSUPPORTED
    size = B.reflex_block_norm_workspace_size
    assert size(4, 16385) == 0 and size(-1, 8) == 0 and size(4, 0) == 0
    assert 0 < size(0, 2048) <= size(4, 2048) <= size(1 << 20, 2048) <= size(1 << 40, 2048)
    need = size(4, 100)
    for changes in (dict(workspace=None), dict(workspace=P + 64), dict(ws_bytes=need - 1)):
        assert call(B.reflex_block_norm_backward, NORM_GRAD, **changes) == B.REFLEX_EWORKSPACE
    # no rows: nothing is looked at but the shapes
    assert call(B.reflex_block_norm, NORM, rows=0, h=None, y=None, out=None,
                norm=None) == B.REFLEX_OK


PLAN = dict(ids=P, k=None, T=4, E=8, k_max=4, cap_rows=16, row_of=P, counts=P, offsets=P, perm=P,
            dev_status=P, workspace=P, ws_bytes=P)


@pytest.mark.parametrize("changes", [
    dict(T=-1), dict(E=0), dict(E=1025), dict(k_max=0), dict(k_max=33), dict(T=(1 << 28) + 1),
    dict(cap_rows=-1)] + [{n: None} for n in ("ids", "row_of", "counts", "offsets")] +
    [{n: P + 2} for n in ("ids", "k", "row_of", "counts", "offsets", "perm", "dev_status")])
def test_plan_refuses(B, changes):
    assert call(B.reflex_expert_plan, PLAN, **changes) == B.REFLEX_EINVAL


def test_plan_workspace(B):
    size = B.reflex_expert_plan_workspace_size
    assert size(4, 1025, 4) == 0 and size(4, 8, 33) == 0 and size(-1, 8, 4) == 0
    assert 0 < size(0, 8, 4) <= size(4, 8, 4) < size(100000, 8, 4) < size(100000, 64, 4)
    sizes = [size(t, 64, 12) for t in range(0, 40000, 97)]
    assert sizes == sorted(sizes)
    for changes in (dict(workspace=None), dict(workspace=P + 64), dict(ws_bytes=size(4, 8, 4) - 1)):
        assert call(B.reflex_expert_plan, PLAN, **changes) == B.REFLEX_EWORKSPACE


ROWS = dict(dtype=1, x=P, ldx=100, row_of=P, T=4, d=100, k_max=4, cap_rows=16, rows=P, ldr=100)
COMBINE = dict(dtype=1, rows=P, ldr=100, alpha=P, row_of=P, residual=P, ldres=100, T=4, d=100,
               k_max=4, cap_rows=16, out=P, ldo=100)
COMBINE_GRAD = dict(dtype=1, d_out=P, ld_d_out=100, rows=P, ldr=100, alpha=P, row_of=P, T=4, d=100,
                    k_max=4, cap_rows=16, d_rows=P, ld_d_rows=100, d_alpha=P)
BAD_ROWS = [dict(dtype=2), dict(T=-1), dict(d=0), dict(k_max=0), dict(k_max=33),
            dict(cap_rows=-1), dict(cap_rows=1 << 31), dict(T=(1 << 28) + 1), dict(row_of=None),
            dict(row_of=P + 2), dict(rows=None), dict(ldr=99), dict(rows=P + 1),
            dict(dtype=0, rows=P + 2)]


@pytest.mark.parametrize("changes", BAD_ROWS + [dict(x=None), dict(ldx=99), dict(x=P + 1)])
def test_rows_refuse(B, changes):
    assert call(B.reflex_expert_rows, ROWS, **changes) == B.REFLEX_EINVAL


@pytest.mark.parametrize("changes", BAD_ROWS + [
    dict(alpha=P + 2), dict(residual=P + 1), dict(ldres=99), dict(out=None), dict(ldo=99),
    dict(out=P + 1)])
def test_combine_refuses(B, changes):
    assert call(B.reflex_expert_combine, COMBINE, **changes) == B.REFLEX_EINVAL


@pytest.mark.parametrize("changes", BAD_ROWS + [
    dict(alpha=None), dict(alpha=P + 2), dict(d_out=None), dict(ld_d_out=99), dict(d_out=P + 1),
    dict(d_rows=None, d_alpha=None), dict(ld_d_rows=99), dict(d_rows=P + 1), dict(d_alpha=P + 2)])
def test_combine_backward_refuses(B, changes):
    assert call(B.reflex_expert_combine_backward, COMBINE_GRAD, **changes) == B.REFLEX_EINVAL


def test_no_tokens(B):
    none = dict(T=0, row_of=None)
    assert call(B.reflex_expert_rows, ROWS, x=None, rows=None, **none) == B.REFLEX_OK
    assert call(B.reflex_expert_combine, COMBINE, rows=None, out=None, **none) == B.REFLEX_OK
    assert call(B.reflex_expert_combine_backward, COMBINE_GRAD, d_out=None, rows=None,
                d_rows=None, d_alpha=None, **none) == B.REFLEX_OK


HEAD = dict(hidden=P, ld_hidden=100, w=P, ldw=104, targets=P, rows=4, vocab=50, k=100, loss=P,
            lse=P, dev_status=P, workspace=P, ws_bytes=1 << 40)
HEAD_GRAD = dict(hidden=P, ld_hidden=100, w=P, ldw=104, targets=P, lse=P, grad=P, rows=4, vocab=50,
                 k=100, d_hidden_dtype=1, d_hidden=P, ld_d_hidden=100, d_w_dtype=1, d_w=P,
                 ld_d_w=100, dev_status=P, workspace=P, ws_bytes=1 << 40)
BAD_HEAD = [dict(rows=-1), dict(vocab=0), dict(k=0), dict(hidden=None), dict(hidden=P + 1),
            dict(ld_hidden=99), dict(w=None), dict(w=P + 8), dict(ldw=96), dict(ldw=101),
            dict(targets=None), dict(targets=P + 2), dict(lse=None), dict(lse=P + 2),
            dict(dev_status=P + 2)]


@pytest.mark.parametrize("changes", BAD_HEAD + [dict(loss=None), dict(loss=P + 2)])
def test_head_loss_refuses(B, changes):
    assert call(B.reflex_head_loss, HEAD, **changes) == B.REFLEX_EINVAL


@pytest.mark.parametrize("changes", BAD_HEAD + [
    dict(grad=None), dict(grad=P + 2), dict(d_hidden=None, d_w=None), dict(d_hidden_dtype=2),
    dict(d_w_dtype=2), dict(ld_d_hidden=99), dict(ld_d_w=99), dict(d_hidden=P + 1),
    dict(d_w=P + 1), dict(d_hidden_dtype=0, d_hidden=P + 2), dict(d_w_dtype=0, d_w=P + 2)])
def test_head_loss_backward_refuses(B, changes):
    assert call(B.reflex_head_loss_backward, HEAD_GRAD, **changes) == B.REFLEX_EINVAL


def test_head_loss_sizes_and_workspace(B):
    huge = (1 << 24) + 1
    for fn, good, size in ((B.reflex_head_loss, HEAD, B.reflex_head_loss_workspace_size),
                           (B.reflex_head_loss_backward, HEAD_GRAD,
                            B.reflex_head_loss_backward_workspace_size)):
        for changes in (dict(rows=huge), dict(vocab=huge), dict(rows=1 << 24, vocab=1 << 24)):
            assert call(fn, good, **changes) == B.REFLEX_EUNSUPPORTED
            assert size(*({**good, **changes}[n] for n in ("rows", "vocab", "k"))) == 0
        need = size(4, 50, 100)
        assert 0 < need < size(4, 5000, 100)
        for changes in (dict(workspace=None), dict(workspace=P + 64), dict(ws_bytes=need - 1)):
            assert call(fn, good, **changes) == B.REFLEX_EWORKSPACE
