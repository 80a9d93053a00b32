"""Torch-facing convenience over the 8-bit entry points: quantisation, the
dense layer and the routed experts.  Codes are torch.float8_e4m3fn tensors,
scales fp32; a scale covers 128 columns of a row (activations) or a 128 x 128
block (weights).  Every step runs in libreflex.so's kernels.  With a `stream`, new
outputs belong to it: to use them on another, wait for it, as torch's own rules have it.
"""
from __future__ import annotations

import torch

from . import _binding as B

_DTYPES = {torch.float32: B.REFLEX_DTYPE_F32, torch.bfloat16: B.REFLEX_DTYPE_BF16}


def _blocks(n: int) -> int:
    return -(-n // 128)


def _want(ok: bool, what: str):
    if not ok:
        raise ValueError(what)


def _new(shape, dtype: torch.dtype, device, stream=None) -> torch.Tensor:
    """An empty tensor in the memory of the stream that writes it: what another stream
    has freed may still be in use there."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream, device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _matrix(t: torch.Tensor, what: str, dtypes):
    """(rows, columns, row stride) of a device matrix whose rows are contiguous,
    any row stride; of one row, its length."""
    if not (t.is_cuda and t.dim() == 2 and t.dtype in dtypes):
        raise ValueError(f"{what}: a CUDA matrix of " + " or ".join(str(d) for d in dtypes))
    rows, cols = t.shape
    ld, step = t.stride()
    if cols > 1 and step != 1:
        raise ValueError(f"{what}: rows must be contiguous")
    if rows <= 1:
        ld = cols
    elif ld < cols:
        raise ValueError(f"{what}: rows must not overlap")
    return rows, cols, ld


def _status_word(status: torch.Tensor | None, device):
    """Refuses an error word that a kernel on `device` could not write."""
    _want(status is None or (status.dtype == torch.int32 and status.numel() == 1
                             and status.device == device),
          "status: one int32 on the device of the inputs")


_F32 = (torch.float32,)
_E4M3 = (torch.float8_e4m3fn,)


def quantize_fp8(x: torch.Tensor, block_rows: int = 1, codes: torch.Tensor | None = None,
                 scales: torch.Tensor | None = None, stream=None):
    """reflex_quantize_fp8 of x [rows, cols] (fp32 or bf16) -> (codes [rows,
    cols] float8_e4m3fn, scales [ceil(rows / block_rows), ceil(cols / 128)]).
    New codes have rows on 16-byte boundaries, as the products take them."""
    rows, cols, ldx = _matrix(x, "x", _DTYPES)
    _want(block_rows in (1, 128), "block_rows is 1 or 128")
    shape = -(-rows // block_rows), _blocks(cols)
    if codes is None:
        ldc = -(-cols // 16) * 16
        codes = _new((rows, ldc), torch.float8_e4m3fn, x.device, stream)
        if ldc != cols:
            codes = codes[:, :cols]
    else:
        r, c, ldc = _matrix(codes, "codes", _E4M3)
        _want((r, c) == (rows, cols), "codes: another shape than x")
        _want(codes.device == x.device, "tensors on several devices")
    if scales is None:
        scales = _new(shape, torch.float32, x.device, stream)
        lds = shape[1]
    else:
        r, c, lds = _matrix(scales, "scales", _F32)
        _want((r, c) == shape, "scales: shape")
        _want(scales.device == x.device, "tensors on several devices")
    B.reflex_quantize_fp8(_DTYPES[x.dtype], x, rows, cols, ldx, block_rows, codes, ldc, scales,
                          lds, stream)
    return codes, scales


def _codes(codes: torch.Tensor, what: str):
    """(rows, columns, row stride) of codes as the products take them; the stride
    of a single row is its length in whole 16-byte vectors."""
    rows, cols, ld = _matrix(codes, what, _E4M3)
    if rows <= 1:
        ld = -(-cols // 16) * 16
    _want(ld % 16 == 0 and codes.data_ptr() % 16 == 0,
          f"{what}: rows start on 16-byte boundaries (as quantize_fp8 lays them out)")
    return rows, cols, ld


def matmul_fp8(a: torch.Tensor, a_scales: torch.Tensor, b: torch.Tensor, b_scales: torch.Tensor,
               out: torch.Tensor | None = None, out_dtype: torch.dtype = torch.bfloat16,
               status: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """reflex_matmul_fp8: A B^T of codes a [M, K] (scales per row and 128
    columns) and b [N, K] (scales per 128 x 128 block) -> [M, N]."""
    M, K, lda = _codes(a, "a")
    N, kb, ldb = _codes(b, "b")
    _want(kb == K, "a and b disagree on K")
    ra, ca, ldas = _matrix(a_scales, "a_scales", _F32)
    rb, cb, ldbs = _matrix(b_scales, "b_scales", _F32)
    _want((ra, ca) == (M, _blocks(K)), "a_scales: shape")
    _want((rb, cb) == (_blocks(N), _blocks(K)), "b_scales: shape")
    _want(a.device == a_scales.device == b.device == b_scales.device,
          "tensors on several devices")
    _status_word(status, a.device)
    out, ldo = _output(out, M, N, out_dtype, a.device, stream)
    B.reflex_matmul_fp8(a, lda, a_scales, ldas, b, ldb, b_scales, ldbs, M, N, K,
                        _DTYPES[out.dtype], out, ldo, status, stream)
    return out


def _output(out, M: int, N: int, dtype, device, stream):
    """The output (given, or new) and its row stride."""
    if out is not None:
        r, c, ldo = _matrix(out, "out", _DTYPES)
        _want((r, c) == (M, N) and out.device == device, "out: shape or device")
        return out, ldo
    _want(dtype in _DTYPES, "outputs are fp32 or bf16")
    # rows on 16-byte boundaries, where a row is a few vectors long at least
    # (999 x 50001 x 2048 to bf16: 99 us, packed rows 229)
    unit = 16 // dtype.itemsize
    ldo = -(-N // unit) * unit if N >= 4 * unit else N
    out = _new((M, ldo), dtype, device, stream)
    return (out if ldo == N else out[:, :N]), ldo


class LinearFp8:
    """A dense layer x W^T in 8 bits with its workspace sized for `max_rows`
    rows: codes [N, K] and scales [ceil(N / 128), ceil(K / 128)] of the weights
    (quantize_fp8 with block_rows 128)."""

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, *, max_rows: int,
                 out_dtype: torch.dtype = torch.bfloat16):
        self.codes, self.scales = codes, scales
        self.N, self.K, self._w_ld = _codes(codes, "codes")
        r, c, self._s_ld = _matrix(scales, "scales", _F32)
        _want((r, c) == (_blocks(self.N), _blocks(self.K)), "scales: shape")
        _want(scales.device == codes.device, "tensors on several devices")
        _want(out_dtype in _DTYPES, "outputs are fp32 or bf16")
        self.max_rows, self.out_dtype = max_rows, out_dtype
        self.ws_bytes = B.reflex_linear_fp8_workspace_size(max_rows, self.K)
        _want(self.ws_bytes > 0, "unsupported shape")
        self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=codes.device)

    def forward(self, x: torch.Tensor, out: torch.Tensor | None = None, stream=None,
                check: bool = True) -> torch.Tensor:
        """x [M, K] fp32 or bf16 -> [M, N] of the layer's output type (or out's)."""
        M, K, ldx = _matrix(x, "x", _DTYPES)
        _want(K == self.K, "x: another number of columns than the weights")
        _want(x.device == self.ws.device, "x is on another device than the weights")
        _want(M <= self.max_rows, "more rows than the workspace was sized for")
        out, ldo = _output(out, M, self.N, self.out_dtype, x.device, stream)
        B.reflex_linear_fp8(_DTYPES[x.dtype], x, ldx, self.codes, self._w_ld, self.scales,
                            self._s_ld, M, self.N, K, _DTYPES[out.dtype], out, ldo, self.ws,
                            self.ws_bytes, stream, check)
        return out

    def status(self, stream=None) -> int:
        return B.reflex_moe_status(self.ws, stream)


def quantize_experts(w_gate_up: torch.Tensor, w_down: torch.Tensor, stream=None) -> dict:
    """The experts' weights w_gate_up [E, 2 inter, d] and w_down [E, d, inter]
    (fp32 or bf16) in 128 x 128 blocks, for ExpertsFp8.  Gate rows and up rows
    are blocked by themselves."""
    e, two, d = (int(n) for n in w_gate_up.shape)
    inter = two // 2
    _want(two == 2 * inter and tuple(w_down.shape) == (e, d, inter), "weights: shapes")
    dev = w_gate_up.device
    gu = _new((e, 2 * inter, d), torch.float8_e4m3fn, dev, stream)
    dn = _new((e, d, inter), torch.float8_e4m3fn, dev, stream)
    gus = _new((e, 2, _blocks(inter), _blocks(d)), torch.float32, dev, stream)
    dns = _new((e, _blocks(d), _blocks(inter)), torch.float32, dev, stream)
    for i in range(e):
        for h in range(2):
            part = slice(h * inter, (h + 1) * inter)
            quantize_fp8(w_gate_up[i, part], 128, gu[i, part], gus[i, h], stream)
        quantize_fp8(w_down[i], 128, dn[i], dns[i], stream)
    return dict(w_gate_up=gu, w_gate_up_scales=gus, w_down=dn, w_down_scales=dns)


class ExpertsFp8:
    """The routed SwiGLU experts of one layer in 8 bits (weights as
    quantize_experts gives them), for a routing that the caller holds; the
    workspace is sized for `max_tokens` tokens at `k_max`."""

    def __init__(self, weights: dict, *, d: int, E: int, inter: int, k_max: int,
                 max_tokens: int):
        self.w, self.d, self.E, self.inter = weights, d, E, inter
        self.k_max, self.max_tokens = k_max, max_tokens
        self.ws_bytes = B.reflex_experts_fp8_workspace_size(max_tokens, d, E, inter, k_max)
        _want(self.ws_bytes > 0, "unsupported MoE layer shape")
        self.check_weights(weights)
        self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=weights["w_down"].device)

    def check_weights(self, weights: dict):
        """Refuses weights that this layer's shape does not fit; `w` may be set to
        others of the same shape (layers that share the workspace)."""
        d, E, inter = self.d, self.E, self.inter
        shapes = dict(w_gate_up=(E, 2 * inter, d), w_down=(E, d, inter),
                      w_gate_up_scales=(E, 2, _blocks(inter), _blocks(d)),
                      w_down_scales=(E, _blocks(d), _blocks(inter)))
        for name, shape in shapes.items():
            t = weights[name]
            dt = torch.float32 if name.endswith("scales") else torch.float8_e4m3fn
            _want(t.is_cuda and t.dtype == dt and tuple(t.shape) == shape and t.is_contiguous()
                  and t.device == weights["w_down"].device,
                  f"{name}: a contiguous CUDA tensor {shape} of {dt}, all on one device")

    def forward(self, hidden: torch.Tensor, ids: torch.Tensor, alpha: torch.Tensor,
                k: torch.Tensor, out: torch.Tensor | None = None, residual: bool = False,
                stream=None, check: bool = True) -> torch.Tensor:
        """hidden [T, d] bf16, ids int32 / alpha fp32 [T, k_max], k int32 [T]
        -> [T, d] bf16 (hidden + experts with residual)."""
        T = int(hidden.shape[0])
        _want(T <= self.max_tokens, "more tokens than the workspace was sized for")
        if out is None:
            out = _new((T, self.d), torch.bfloat16, hidden.device, stream)
        for t, dt, shape, what in ((hidden, torch.bfloat16, (T, self.d), "hidden"),
                                   (ids, torch.int32, (T, self.k_max), "ids"),
                                   (alpha, torch.float32, (T, self.k_max), "alpha"),
                                   (k, torch.int32, (T,), "k"),
                                   (out, torch.bfloat16, (T, self.d), "out")):
            _want(t.is_cuda and t.dtype == dt and tuple(t.shape) == shape and t.is_contiguous()
                  and t.device == self.ws.device,
                  f"{what}: a contiguous {shape} tensor of {dt} on the weights' device")
        B.reflex_experts_fp8(hidden, ids, alpha, k, self.w["w_gate_up"],
                             self.w["w_gate_up_scales"], self.w["w_down"],
                             self.w["w_down_scales"], T, self.d, self.E, self.inter, self.k_max,
                             B.REFLEX_FLAG_RESIDUAL if residual else 0, self.ws, self.ws_bytes,
                             out, stream, check)
        return out

    def status(self, stream=None) -> int:
        return B.reflex_moe_status(self.ws, stream)
