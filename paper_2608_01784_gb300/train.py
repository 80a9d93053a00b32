"""Torch-facing convenience over the entry points around the experts that have
gradients: norms around a block, tokens to experts and back, the loss of a head.  A
gradient is a call of its own (no autograd graph is kept), takes the forward call's
inputs again and allocates only what it returns and a workspace, so each can be
captured in a CUDA graph.  With a `stream`, new outputs belong to it: to use them on
another, wait for it, as torch's own rules have it.
"""
from __future__ import annotations

import torch

from . import _binding as B
from .fp8 import _DTYPES, _matrix, _new, _status_word, _want


_MOST = 2 ** 31 - 1  # of a size that the library takes in 32 bits


def _here(device):
    """A launch goes to the current device; tensors of another one are refused."""
    if device.index != B.current_device():
        raise ValueError("the tensors are on another device than the current one")


def _new_like(t: torch.Tensor, stream) -> torch.Tensor:
    """An empty contiguous tensor like t, as _new has it (0.4 us less where t allows)."""
    if stream is None and t.is_contiguous():
        return torch.empty_like(t)
    return _new(tuple(t.shape), t.dtype, t.device, stream)


def _like(t: torch.Tensor, x: torch.Tensor, what: str) -> int:
    """The row stride of t, which has x's shape, type and device."""
    if t.shape != x.shape or t.dtype is not x.dtype or t.device != x.device:
        raise ValueError(f"{what}: shape, type or device")
    return x.shape[1] if t.is_contiguous() else _matrix(t, what, _DTYPES)[2]


def _rows(t: torch.Tensor, rows: int, dtype, device, what: str):
    if not (t.dtype is dtype and t.shape == (rows,) and t.is_contiguous() and t.device == device):
        raise ValueError(f"{what}: {rows} contiguous values of {dtype}")


def _vector(t: torch.Tensor | None, d: int, x: torch.Tensor, what: str):
    if t is not None and not (t.dtype is x.dtype and t.shape == (d,) and t.is_contiguous()
                              and t.device == x.device):
        raise ValueError(f"{what}: {d} contiguous values of the stream's type on its device")


def _norm_inputs(h, y, w_after, w_before, gate):
    """Checks them; (rows, d, ldh, ldy, ldg)."""
    rows, d, ldh = _matrix(h, "h", _DTYPES)
    if not 1 <= d <= _MOST:
        raise ValueError("h: no columns, or an unsupported width")
    _here(h.device)
    if y is not None:
        ldy = _like(y, h, "y")
    elif w_after is not None or gate is not None:
        raise ValueError("w_after and gate need y")
    else:
        ldy = 0
    _vector(w_after, d, h, "w_after")
    _vector(w_before, d, h, "w_before")
    if gate is not None and gate.dim() == 2:
        return rows, d, ldh, ldy, _like(gate, h, "gate")
    _vector(gate, d, h, "gate")
    return rows, d, ldh, ldy, 0


def block_norm(h: torch.Tensor, y: torch.Tensor | None = None, *,
               w_after: torch.Tensor | None = None, w_before: torch.Tensor | None = None,
               gate: torch.Tensor | None = None, scale: float = 1.0, eps: float = 1e-6,
               out: torch.Tensor | None = None, norm: torch.Tensor | None = None, stream=None):
    """reflex_block_norm: (h + scale * gate * norm(y) w_after, its own norm times
    w_before).  h, y [rows, d] fp32 or bf16, gate [d] or [rows, d]; without w_after
    y is not normalised, without y the stream is h itself, without w_before the
    second value is None.  `out` and `norm` may be h or y."""
    rows, d, ldh, ldy, ldg = _norm_inputs(h, y, w_after, w_before, gate)
    ldo = ldn = d
    if out is None:
        out = _new_like(h, stream)
    else:
        ldo = _like(out, h, "out")
    if norm is not None:
        _want(w_before is not None, "norm needs w_before")
        ldn = _like(norm, h, "norm")
    elif w_before is not None:
        norm = _new_like(h, stream)
    B.reflex_block_norm(_DTYPES[h.dtype], h, ldh, y, ldy, w_after, gate, ldg, w_before, scale, eps,
                        rows, d, out, ldo, norm, ldn, stream)
    return out, norm


def block_norm_backward(h: torch.Tensor, y: torch.Tensor | None, d_out: torch.Tensor | None,
                        d_norm: torch.Tensor | None, *, w_after: torch.Tensor | None = None,
                        w_before: torch.Tensor | None = None, gate: torch.Tensor | None = None,
                        scale: float = 1.0, eps: float = 1e-6, d_h: torch.Tensor | None = None,
                        d_y: torch.Tensor | None = None, stream=None) -> dict:
    """reflex_block_norm_backward: the gradients of block_norm's inputs from those of
    its outputs (d_out may be None; d_norm comes with w_before), as a dict of "h", "y",
    "gate", "w_after" and "w_before", None for inputs that are not given.  `d_h` and
    `d_y` may be any [rows, d] input."""
    rows, d, ldh, ldy, ldg = _norm_inputs(h, y, w_after, w_before, gate)
    _want((d_norm is not None) == (w_before is not None), "d_norm comes with w_before")
    _want(d_out is not None or d_norm is not None, "no gradient of an output")
    _want(d_y is None or y is not None, "d_y needs y")
    ld_d_out = _like(d_out, h, "d_out") if d_out is not None else 0
    ld_d_norm = _like(d_norm, h, "d_norm") if d_norm is not None else 0

    def new(like):
        return None if like is None else _new_like(like, stream)
    ld_d_h = _like(d_h, h, "d_h") if d_h is not None else d
    ld_d_y = _like(d_y, h, "d_y") if d_y is not None else d
    got = dict(w_after=new(w_after), w_before=new(w_before), gate=new(gate),
               h=new(h) if d_h is None else d_h, y=new(y) if d_y is None else d_y)
    ws_bytes = B.reflex_block_norm_workspace_size(rows, d)
    _want(ws_bytes > 0, "unsupported width")
    ws = _new(ws_bytes, torch.uint8, h.device, stream)
    B.reflex_block_norm_backward(_DTYPES[h.dtype], h, ldh, y, ldy, w_after, gate, ldg, w_before,
                                 scale, eps, rows, d, d_out, ld_d_out, d_norm, ld_d_norm,
                                 got["h"], ld_d_h, got["y"], ld_d_y, got["gate"], d,
                                 got["w_after"], got["w_before"], ws, ws_bytes, stream)
    return got


class ExpertPlan:
    """Where the pairs of a routing lie in expert order (reflex_expert_plan): row_of
    int32 [T, k_max], counts [E], offsets [E + 1], all on the device; the pairs' rows
    are 0 .. offsets[E] - 1 of at most cap_rows.  One allocation holds them all; the
    tensors are views of it."""

    def __init__(self, T: int, E: int, k_max: int, cap_rows: int, device, stream=None):
        self.T, self.E, self.k_max, self.cap_rows = T, E, k_max, cap_rows
        fits = E <= _MOST and k_max <= _MOST
        self.ws_bytes = B.reflex_expert_plan_workspace_size(T, E, k_max) if fits else 0
        if self.ws_bytes == 0:
            raise ValueError("unsupported shape: E up to 1024, k_max up to 32")
        # the workspace, then row_of, counts, offsets and the error word
        self._at = at = self.ws_bytes // 4
        self._words = _new(at + T * k_max + 2 * E + 2, torch.int32, device, stream)
        self.device = device
        self.ws = base = self._words.data_ptr()
        self.row_of_ptr = base + 4 * at
        self.counts_ptr = self.row_of_ptr + 4 * T * k_max
        self.offsets_ptr = self.counts_ptr + 4 * E
        self.error_ptr = self.offsets_ptr + 4 * (E + 1)

    @property
    def row_of(self) -> torch.Tensor:
        return self._words.as_strided((self.T, self.k_max), (self.k_max, 1), self._at)

    @property
    def counts(self) -> torch.Tensor:
        return self._words.as_strided((self.E,), (1,), self._at + self.T * self.k_max)

    @property
    def offsets(self) -> torch.Tensor:
        return self._words.as_strided((self.E + 1,), (1,),
                                      self._at + self.T * self.k_max + self.E)

    def status(self, stream=None) -> int:
        """What the last plan found wrong with its routing (waits)."""
        return B.reflex_read_status(self.error_ptr, stream)


def expert_plan(ids: torch.Tensor, *, E: int, k: torch.Tensor | None = None,
                cap_rows: int | None = None, plan: ExpertPlan | None = None,
                perm: torch.Tensor | None = None, stream=None) -> ExpertPlan:
    """reflex_expert_plan of ids int32 [T, k_max]: slots j < k[t] are used, or, without
    k, those with ids >= 0.  `plan` (of the same T, E, k_max and cap_rows) is filled
    again instead of a new one; `perm` int32 [T * k_max] receives row -> t * k_max + j."""
    if not (ids.is_cuda and ids.dim() == 2 and ids.dtype is torch.int32 and ids.is_contiguous()):
        raise ValueError("ids: a contiguous CUDA matrix of torch.int32")
    dev = ids.device
    _here(dev)
    T, k_max = ids.shape
    for t, n, what in ((k, T, "k"), (perm, T * k_max, "perm")):
        if t is not None:
            _rows(t, n, torch.int32, dev, what)
    if plan is None:
        plan = ExpertPlan(T, E, k_max, T * k_max if cap_rows is None else cap_rows, dev, stream)
    else:
        _want((plan.T, plan.E, plan.k_max) == (T, E, k_max) and plan.device == dev
              and cap_rows in (None, plan.cap_rows), "plan: made for another shape or device")
    B.reflex_expert_plan(ids, k, T, E, k_max, plan.cap_rows, plan.row_of_ptr, plan.counts_ptr,
                         plan.offsets_ptr, perm, plan.error_ptr, plan.ws, plan.ws_bytes, stream)
    return plan


def _pair_rows(rows: torch.Tensor, plan: ExpertPlan, what: str):
    """(d, row stride) of the pairs' rows of a plan."""
    n, d, ld = _matrix(rows, what, _DTYPES)
    if n < plan.cap_rows or not 1 <= d <= _MOST or rows.device != plan.device:
        raise ValueError(f"{what}: fewer rows than the plan's cap_rows, no columns or too many, or "
                         "another device")
    _here(plan.device)
    return d, ld


def _tokens(x: torch.Tensor, plan: ExpertPlan, d: int, dtype, what: str) -> int:
    rows, cols, ld = _matrix(x, what, (dtype,))
    if (rows, cols) != (plan.T, d) or x.device != plan.device:
        raise ValueError(f"{what}: a row for each of the plan's tokens, of the rows' width and "
                         "device")
    return ld


def _weights(alpha: torch.Tensor, plan: ExpertPlan, what: str):
    if not (alpha.dtype is torch.float32 and alpha.shape == (plan.T, plan.k_max)
            and alpha.is_contiguous() and alpha.device == plan.device):
        raise ValueError(f"{what}: a contiguous tensor of torch.float32 of the plan's [T, k_max]")


def expert_rows(x: torch.Tensor, plan: ExpertPlan, *, rows: torch.Tensor | None = None,
                stream=None) -> torch.Tensor:
    """reflex_expert_rows: x [T, d] (fp32 or bf16) laid out by expert, [cap_rows, d].
    `rows` behind the last pair are left as they are; of a new tensor they are not set."""
    if rows is None:
        rows = _new((plan.cap_rows, x.shape[-1]), x.dtype, x.device, stream)
    d, ldr = _pair_rows(rows, plan, "rows")
    ldx = _tokens(x, plan, d, rows.dtype, "x")
    B.reflex_expert_rows(_DTYPES[x.dtype], x, ldx, plan.row_of_ptr, plan.T, d, plan.k_max,
                         plan.cap_rows, rows, ldr, stream)
    return rows


def _sum(rows, alpha, plan, residual, out, stream):
    d, ldr = _pair_rows(rows, plan, "rows")
    ldres = _tokens(residual, plan, d, rows.dtype, "residual") if residual is not None else 0
    ldo = d
    if out is None:
        out = (_new_like(residual, stream) if residual is not None else
               _new((plan.T, d), rows.dtype, rows.device, stream))
    else:
        ldo = _tokens(out, plan, d, rows.dtype, "out")
    B.reflex_expert_combine(_DTYPES[rows.dtype], rows, ldr, alpha, plan.row_of_ptr, residual, ldres,
                            plan.T, d, plan.k_max, plan.cap_rows, out, ldo, stream)
    return out


def expert_rows_backward(d_rows: torch.Tensor, plan: ExpertPlan, *,
                         out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """The gradient of expert_rows' x from that of its rows: their sums by token."""
    return _sum(d_rows, None, plan, None, out, stream)


def expert_combine(rows: torch.Tensor, alpha: torch.Tensor, plan: ExpertPlan, *,
                   residual: torch.Tensor | None = None, out: torch.Tensor | None = None,
                   stream=None) -> torch.Tensor:
    """reflex_expert_combine: out[t] = sum_j alpha[t, j] rows[row_of[t, j]] (+ residual[t]);
    alpha fp32 [T, k_max].  `out` may be residual."""
    _weights(alpha, plan, "alpha")
    return _sum(rows, alpha, plan, residual, out, stream)


def expert_combine_backward(d_out: torch.Tensor, rows: torch.Tensor, alpha: torch.Tensor,
                            plan: ExpertPlan, *, d_rows: torch.Tensor | None = None,
                            d_alpha: torch.Tensor | None = None, stream=None):
    """reflex_expert_combine_backward: (gradient of the rows, of alpha); that of the
    residual is d_out.  `d_rows` may be rows; behind the last pair it is left as it is."""
    d, ldr = _pair_rows(rows, plan, "rows")
    ldd = _tokens(d_out, plan, d, rows.dtype, "d_out")
    _weights(alpha, plan, "alpha")
    if d_alpha is None:
        d_alpha = _new_like(alpha, stream)
    else:
        _weights(d_alpha, plan, "d_alpha")
    lddr = d
    if d_rows is None:
        d_rows = _new((plan.cap_rows, d), rows.dtype, rows.device, stream)
    else:
        dd, lddr = _pair_rows(d_rows, plan, "d_rows")
        _want(dd == d and d_rows.dtype == rows.dtype, "d_rows: another width or type than rows")
    B.reflex_expert_combine_backward(_DTYPES[rows.dtype], d_out, ldd, rows, ldr, alpha,
                                     plan.row_of_ptr, plan.T, d, plan.k_max, plan.cap_rows, d_rows,
                                     lddr, d_alpha, stream)
    return d_rows, d_alpha


_BF16 = (torch.bfloat16,)


def _head(hidden, weight, targets, status):
    """Checks them; (rows, vocab, k, ld_hidden, ldw)."""
    rows, k, ld_hidden = _matrix(hidden, "hidden", _BF16)
    vocab, kw, ldw = _matrix(weight, "weight", _BF16)
    if k < 1 or vocab < 1 or kw != k:
        raise ValueError("hidden and weight disagree on their columns, or have none")
    _want(max(rows, vocab, k) <= _MOST, "unsupported sizes")
    if vocab == 1:
        ldw = -(-k // 8) * 8
    if ldw % 8 or weight.data_ptr() % 16:
        raise ValueError("weight: rows start on 16-byte boundaries")
    dev = hidden.device
    if dev != weight.device:
        raise ValueError("tensors on several devices")
    _here(dev)
    _rows(targets, rows, torch.int32, dev, "targets")
    if status is not None:
        _status_word(status, dev)
    return rows, vocab, k, ld_hidden, ldw


def head_loss(hidden: torch.Tensor, weight: torch.Tensor, targets: torch.Tensor, *,
              loss: torch.Tensor | None = None, lse: torch.Tensor | None = None,
              status: torch.Tensor | None = None, stream=None):
    """reflex_head_loss: (loss, lse) fp32 [rows] of the softmax of hidden weight^T at
    targets int32 [rows], zeros where a target is negative.  hidden [rows, k] and weight
    [vocab, k] are bf16; the logits are not kept."""
    rows, vocab, k, ld_hidden, ldw = _head(hidden, weight, targets, status)
    dev = hidden.device
    if loss is None:
        loss = _new(rows, torch.float32, dev, stream)
    else:
        _rows(loss, rows, torch.float32, dev, "loss")
    if lse is None:
        lse = _new(rows, torch.float32, dev, stream)
    else:
        _rows(lse, rows, torch.float32, dev, "lse")
    ws_bytes = B.reflex_head_loss_workspace_size(rows, vocab, k)
    _want(ws_bytes > 0, "unsupported sizes")
    ws = _new(ws_bytes, torch.uint8, dev, stream)
    B.reflex_head_loss(hidden, ld_hidden, weight, ldw, targets, rows, vocab, k, loss, lse, status,
                       ws, ws_bytes, stream)
    return loss, lse


def _gradient(out, rows: int, cols: int, device, stream, what: str):
    """A gradient (given, or new in bf16 with rows on 16-byte boundaries) and its stride."""
    if out is None:
        ld = -(-cols // 8) * 8
        out = _new((rows, ld), torch.bfloat16, device, stream)
        return (out if ld == cols else out[:, :cols]), ld
    r, c, ld = _matrix(out, what, _DTYPES)
    _want((r, c) == (rows, cols) and out.device == device, f"{what}: shape or device")
    return out, ld


def _overlap(a: torch.Tensor, lda: int, b: torch.Tensor, ldb: int) -> bool:
    """Whether two matrices of one width share bytes (as reflex_head_loss_backward has it:
    rows of one stride may lie between one another, ranges of different ones that cross
    count as shared)."""
    (rows, cols), rows_b = a.shape, b.shape[0]
    if rows == 0 or rows_b == 0:
        return False
    (pa, pitch, wa), (pb, other, wb) = ((t.data_ptr(), ld * t.element_size(), cols * t.element_size())
                                        for t, ld in ((a, lda), (b, ldb)))
    if pa + (rows - 1) * pitch + wa <= pb or pb + (rows_b - 1) * other + wb <= pa:
        return False
    off = (pb - pa) % pitch
    return pitch != other or off < wa or off + wb > pitch


def head_loss_backward(hidden: torch.Tensor, weight: torch.Tensor, targets: torch.Tensor,
                       lse: torch.Tensor, grad: torch.Tensor, *,
                       d_hidden: torch.Tensor | None = None,
                       d_weight: torch.Tensor | None = None, need_hidden: bool = True,
                       need_weight: bool = True, status: torch.Tensor | None = None,
                       stream=None):
    """reflex_head_loss_backward: the gradients (of hidden, of weight) from grad fp32
    [rows], that of each row's loss, and head_loss's lse.  They come in bf16, or in the
    type of `d_hidden` and `d_weight` (fp32 or bf16); the one that is not needed is None.
    `d_hidden` may be hidden; neither shares bytes with weight or with the other."""
    rows, vocab, k, ld_hidden, ldw = _head(hidden, weight, targets, status)
    dev = hidden.device
    _rows(lse, rows, torch.float32, dev, "lse")
    _rows(grad, rows, torch.float32, dev, "grad")
    _want(need_hidden or need_weight, "no gradient wanted")
    _want((need_hidden or d_hidden is None) and (need_weight or d_weight is None),
          "a place for a gradient that is not needed")
    ld_dh = ld_dw = k
    dt_h = dt_w = B.REFLEX_DTYPE_BF16
    if need_hidden:
        given_h = d_hidden is not None
        d_hidden, ld_dh = _gradient(d_hidden, rows, k, dev, stream, "d_hidden")
        _want(not given_h or not _overlap(weight, ldw, d_hidden, ld_dh),
              "d_hidden: the weights are still read while it is written")
        dt_h = _DTYPES[d_hidden.dtype]
    if need_weight:
        given = d_weight is not None
        d_weight, ld_dw = _gradient(d_weight, vocab, k, dev, stream, "d_weight")
        _want(not given or not _overlap(weight, ldw, d_weight, ld_dw),
              "d_weight: the weights are still read while it is written")
        _want(not (given and need_hidden) or not _overlap(d_weight, ld_dw, d_hidden, ld_dh),
              "d_hidden and d_weight overlap")
        dt_w = _DTYPES[d_weight.dtype]
    ws_bytes = B.reflex_head_loss_backward_workspace_size(rows, vocab, k)
    _want(ws_bytes > 0, "unsupported sizes")
    ws = _new(ws_bytes, torch.uint8, dev, stream)
    B.reflex_head_loss_backward(hidden, ld_hidden, weight, ldw, targets, lse, grad, rows, vocab, k,
                                dt_h, d_hidden, ld_dh, dt_w, d_weight, ld_dw, status, ws, ws_bytes,
                                stream)
    return d_hidden, d_weight
