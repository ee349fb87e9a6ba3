"""Matrix products in 8-bit floating point (f7 to f9; see include/lazytrain.h) and the linear layer
made of them: weights that the optimizer has just updated are quantized once, read by the
forward and the input-gradient product, and the weight gradient comes back in bfloat16 (or
float32) for the next step.
"""
from __future__ import annotations

import math
from typing import Optional, Tuple

import torch
from torch.autograd.graph import increment_version

from .lazytrain import (LT_DTYPE_BF16, LT_DTYPE_F32, _capturing, _check, _current, _on, _own,
                        _stream_handle, _track, _workspace, lib)

_DTYPES = {torch.float32: LT_DTYPE_F32, torch.bfloat16: LT_DTYPE_BF16}
_BYTES = (torch.uint8, torch.float8_e4m3fn)


def lt_fp8_code_pitch(cols: int) -> int:
    """Bytes of a row of codes of a matrix with `cols` columns."""
    return -(-cols // 128) * 128


def lt_fp8_scale_pitch(cols: int) -> int:
    """Bytes of a row of its scales."""
    return -(-cols // 512) * 4


def _dtype_code(t: torch.Tensor, what: str) -> int:
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"{what} must be float32 or bfloat16, got {t.dtype}")
    return code


def _rows(t: torch.Tensor, what: str) -> int:
    """The row stride of a matrix whose rows are contiguous."""
    if t.dim() != 2:
        raise ValueError(f"{what} must be a matrix (two dimensions, got {t.dim()})")
    rows, cols = t.shape
    if cols > 1 and t.stride(1) != 1:
        raise ValueError(f"{what} must have contiguous rows")
    stride = t.stride(0) if rows > 1 else cols
    if stride < cols:
        raise ValueError(f"{what}: rows must not overlap")
    return stride


def _layout(codes, scales, rows: int, cols: int, device, what: str) -> Tuple[int, int]:
    """Addresses of a layout's codes and scales (0, 0 for none)."""
    if codes is None and scales is None:
        return 0, 0
    if codes is None or scales is None:
        raise ValueError(f"{what} come with their scales")
    for t, pitch, name in ((codes, lt_fp8_code_pitch(cols), what),
                           (scales, lt_fp8_scale_pitch(cols), what + " scales")):
        if t.device != device or t.dtype not in _BYTES or not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous bytes on {device}")
        if t.numel() != rows * pitch:
            raise ValueError(f"{name} must have {rows} rows of {pitch} bytes")
    return codes.data_ptr(), scales.data_ptr()


def _scratch(device, nbytes: int, workspace, stream) -> Tuple[torch.Tensor, int, int]:
    """(tensor, address, bytes) of the caller's workspace, or of memory of this call's own: what
    a call keeps there between its launches is not for another call on the stream to overwrite,
    from another thread or in a graph's replays."""
    if workspace is not None:
        ws = _workspace(device, nbytes, workspace, stream, "fp8")
    else:
        ws = _own(device, nbytes, stream)
        if _capturing(stream, device):
            _track(ws)  # the library notes that a graph writes there
    return ws, ws.data_ptr(), ws.numel() * ws.element_size()


def lt_fp8_quantize(x: torch.Tensor, codes: Optional[torch.Tensor] = None,
                    scales: Optional[torch.Tensor] = None,
                    codes_t: Optional[torch.Tensor] = None,
                    scales_t: Optional[torch.Tensor] = None, square: bool = False,
                    stream=None) -> None:
    """f7: quantizes x (rows, cols; float32 or bfloat16, contiguous rows) into codes and scales
    by rows, and into those of its transpose; either may be left out.  With `square` a scale
    holds for a 128 x 128 block, else for 128 columns of a row."""
    stride = _rows(x, "x")
    rows, cols = x.shape
    code = _dtype_code(x, "x")
    device = x.device
    c, s = _layout(codes, scales, rows, cols, device, "codes")
    ct, st = _layout(codes_t, scales_t, cols, rows, device, "codes_t")
    with _current(device):
        _check(lib().lt_fp8_quantize(x.data_ptr(), code, rows, cols, stride, int(bool(square)), c,
                                     s, ct, st, _stream_handle(stream, device)))
    # autograd's in-place rule: a graph that saved one of these has lost its values
    increment_version([t for t in (codes, scales, codes_t, scales_t) if t is not None])


def lt_fp8_matmul(a_codes: torch.Tensor, a_scales: torch.Tensor, b_codes: torch.Tensor,
                  b_scales: torch.Tensor, k: int, out: torch.Tensor,
                  workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """f8: out[i, j] = sum over k of A[i, k] * B[j, k] for operands that lt_fp8_quantize made;
    out is (m, n), float32 or bfloat16, with contiguous rows."""
    stride = _rows(out, "out")
    m, n = out.shape
    code = _dtype_code(out, "out")
    device = out.device
    a, sa = _layout(a_codes, a_scales, m, k, device, "a_codes")
    b, sb = _layout(b_codes, b_scales, n, k, device, "b_codes")
    ws, nbytes, handle = 0, 0, _stream_handle(stream, device)
    if (m > 32 and k > 512) or workspace is not None:
        nbytes = int(lib().lt_fp8_matmul_workspace_bytes(m, n, k))
        held, ws, nbytes = _scratch(device, nbytes, workspace, stream)
    with _current(device):
        _check(lib().lt_fp8_matmul(a, sa, b, sb, m, n, k, out.data_ptr(), code, stride, ws,
                                   nbytes, handle))


class Fp8Weight:
    """A linear layer's weight (out_features x in_features) in 8-bit floating point, a scale for
    each 128 x 128 block: codes and scales by rows, which the forward product reads, and of
    the transpose, which the input-gradient product reads (None where only answers are
    computed).  ``update`` quantizes the master weights into it again after a step."""

    __slots__ = ("rows", "cols", "codes", "scales", "codes_t", "scales_t")

    def __init__(self, rows: int, cols: int, codes: torch.Tensor, scales: torch.Tensor,
                 codes_t: Optional[torch.Tensor] = None, scales_t: Optional[torch.Tensor] = None):
        self.rows, self.cols = int(rows), int(cols)
        _layout(codes, scales, self.rows, self.cols, codes.device, "codes")
        _layout(codes_t, scales_t, self.cols, self.rows, codes.device, "codes_t")
        self.codes, self.scales, self.codes_t, self.scales_t = codes, scales, codes_t, scales_t

    @classmethod
    def empty(cls, rows: int, cols: int, device, transposed: bool = True) -> "Fp8Weight":
        codes, scales = _empty(rows, cols, device)
        codes_t, scales_t = _empty(cols, rows, device) if transposed else (None, None)
        return cls(rows, cols, codes, scales, codes_t, scales_t)

    @classmethod
    def from_master(cls, w: torch.Tensor, transposed: bool = True) -> "Fp8Weight":
        """Quantizes a weight matrix (float32 or bfloat16) on the current stream."""
        if w.dim() != 2:
            raise ValueError(f"w must be a matrix (two dimensions, got {w.dim()})")
        weight = cls.empty(w.shape[0], w.shape[1], w.device, transposed)
        weight.update(w)
        return weight

    def update(self, w: torch.Tensor, stream=None) -> None:
        if tuple(w.shape) != (self.rows, self.cols):
            raise ValueError(f"w must have shape {(self.rows, self.cols)}")
        with _on(stream, w.device):  # a copy of w belongs to the stream that reads it
            w = _laid_out(w)
            lt_fp8_quantize(w, self.codes, self.scales, self.codes_t, self.scales_t, square=True)


def _empty(rows: int, cols: int, device):
    return (torch.empty(rows, lt_fp8_code_pitch(cols), dtype=torch.uint8, device=device),
            torch.empty(rows, lt_fp8_scale_pitch(cols), dtype=torch.uint8, device=device))


def _laid_out(t: torch.Tensor, aligned: bool = True) -> torch.Tensor:
    """A matrix as the library takes it: rows contiguous and apart, beginning on 16 bytes (not
    `aligned`: anywhere).  Any other is copied: transposed or broadcast tokens, part of a packed
    batch at an odd width."""
    if ((t.shape[1] > 1 and t.stride(1) != 1) or (t.shape[0] > 1 and t.stride(0) < t.shape[1]) or
            (aligned and t.data_ptr() % 16)):
        return t.clone(memory_format=torch.contiguous_format)
    return t


def _tokens(x: torch.Tensor, features: int, what: str, aligned: bool = True) -> torch.Tensor:
    if x.dim() < 1 or x.shape[-1] != features:
        raise ValueError(f"{what} must have {features} features, got shape {tuple(x.shape)}")
    t = x if x.dim() == 2 else x.reshape(math.prod(x.shape[:-1]), features)
    return _laid_out(t, aligned)


def fp8_linear(x: torch.Tensor, weight: Fp8Weight,
               out_dtype: torch.dtype = torch.bfloat16,
               workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """f9: x weight^T for x (..., in_features), quantized on the way; for answering: nothing is
    kept for a backward pass.  This and the functions below allocate and work on the current
    stream."""
    t = _tokens(x, weight.cols, "x", aligned=False)
    stride = _rows(t, "x")
    m, device = t.shape[0], x.device
    if weight.codes.device != device:
        raise ValueError(f"the weight is on {weight.codes.device}, x on {device}")
    y = torch.empty(m, weight.rows, dtype=out_dtype, device=device)
    ws, nbytes, handle = 0, 0, _stream_handle(None, device)
    if m > 16 or workspace is not None:
        nbytes = int(lib().lt_fp8_linear_workspace_bytes(m, weight.rows, weight.cols))
        held, ws, nbytes = _scratch(device, nbytes, workspace, None)
    with _current(device):
        _check(lib().lt_fp8_linear(t.data_ptr(), _dtype_code(t, "x"), stride,
                                   weight.codes.data_ptr(), weight.scales.data_ptr(), m,
                                   weight.rows, weight.cols, y.data_ptr(), _dtype_code(y, "y"),
                                   weight.rows, ws, nbytes, handle))
    return y if x.dim() == 2 else y.view(*x.shape[:-1], weight.rows)


def fp8_linear_forward(x: torch.Tensor, weight: Fp8Weight,
                       out_dtype: torch.dtype = torch.bfloat16):
    """As fp8_linear, and what the backward pass needs of x: its transpose, quantized along the
    tokens (one byte a value)."""
    return _answer(x, weight, out_dtype, True)


def _answer(x, weight: Fp8Weight, out_dtype, keep: bool):
    """y, and x's transpose (codes and scales) where it is to be kept."""
    t = _tokens(x, weight.cols, "x")
    codes, scales = _empty(t.shape[0], weight.cols, x.device)
    saved = _empty(weight.cols, t.shape[0], x.device) if keep else (None, None)
    lt_fp8_quantize(t, codes, scales, *saved)
    y = torch.empty(t.shape[0], weight.rows, dtype=out_dtype, device=x.device)
    lt_fp8_matmul(codes, scales, weight.codes, weight.scales, weight.cols, y)
    return y.view(*x.shape[:-1], weight.rows), saved


def fp8_linear_backward(dy: torch.Tensor, saved, weight: Fp8Weight,
                        out_dtype: torch.dtype = torch.bfloat16,
                        grad_dtype: torch.dtype = torch.bfloat16):
    """(dx, dw) of fp8_linear_forward: dx in out_dtype with dy's leading shape, dw (out_features
    x in_features) in grad_dtype."""
    if weight.codes_t is None:
        raise ValueError("the weight has no transposed codes: the backward pass needs them")
    return _gradients(dy, saved, (weight.codes_t, weight.scales_t), weight.rows, weight.cols,
                      out_dtype, grad_dtype)


def _gradients(dy, saved, transposed, rows: int, cols: int, out_dtype, grad_dtype):
    """dx (None without the weight's transpose) and dw (None without x's) from dy, the operands
    as codes and scales; dy is laid out for what is asked for."""
    t = _tokens(dy, rows, "dy")
    tokens, device = t.shape[0], dy.device
    dx = dw = None
    by_rows = _empty(tokens, rows, device) if transposed is not None else (None, None)
    turned = _empty(rows, tokens, device) if saved is not None else (None, None)
    if transposed is not None or saved is not None:
        lt_fp8_quantize(t, *by_rows, *turned)
    if transposed is not None:
        dx = torch.empty(tokens, cols, dtype=out_dtype, device=device)
        lt_fp8_matmul(*by_rows, *transposed, rows, dx)
        dx = dx.view(*dy.shape[:-1], cols)
    if saved is not None:
        dw = torch.empty(rows, cols, dtype=grad_dtype, device=device)
        lt_fp8_matmul(*turned, *saved, tokens, dw)
    return dx, dw


class Fp8Linear(torch.autograd.Function):
    """``Fp8Linear.apply(x, w, weight)``: x weight^T with gradients for x and for w, the tensor
    (float32 or bfloat16, for instance the optimizer's bf16 copy) that stands for the weight in
    the graph and whose values ``weight`` was quantized from.  The gradient for x reads the
    weight's codes again: once ``weight`` is updated, a backward pass of a forward pass before
    raises, like autograd's own after a change in place.  First derivatives only: a backward
    pass that is itself to be differentiated raises, where its gradients depend on what needs
    one."""

    @staticmethod
    def forward(ctx, x, w, weight):
        if tuple(w.shape) != (weight.rows, weight.cols):
            raise ValueError(f"w must have shape {(weight.rows, weight.cols)}")
        if ctx.needs_input_grad[0] and weight.codes_t is None:
            raise ValueError("the weight has no transposed codes: the gradient for x needs them")
        if ctx.needs_input_grad[1]:
            _dtype_code(w, "w")  # its gradient's
        y, saved = _answer(x, weight, x.dtype, ctx.needs_input_grad[1])
        transposed = ((weight.codes_t, weight.scales_t) if ctx.needs_input_grad[0]
                      else (None, None))
        ctx.save_for_backward(*saved, *transposed)
        ctx.sizes, ctx.w_dtype = (weight.rows, weight.cols), w.dtype
        return y

    @staticmethod
    def backward(ctx, dy):
        # dx depends on dy and w, dw on dy and x, and the products leave no graph
        if torch.is_grad_enabled() and (dy.requires_grad or all(ctx.needs_input_grad[:2])):
            raise RuntimeError("Fp8Linear has first derivatives only: its backward pass cannot be "
                               "part of a graph (create_graph=True)")
        x_t, x_scales_t, w_t, w_scales_t = ctx.saved_tensors
        saved = (x_t, x_scales_t) if ctx.needs_input_grad[1] else None
        transposed = (w_t, w_scales_t) if ctx.needs_input_grad[0] else None
        dx, dw = _gradients(dy, saved, transposed, *ctx.sizes, dy.dtype, ctx.w_dtype)
        return dx, dw, None
