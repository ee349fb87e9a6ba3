"""Matrix products in 8-bit integers with a scale for each token and output channel (f10 to f12; see
include/lazytrain.h), for answering: a linear layer and the gated projections of a feed-forward
block, with weights that are quantized once after the last step.
"""
from __future__ import annotations

from typing import Optional, Tuple

import torch
from torch.autograd.graph import increment_version

from .fp8 import _dtype_code, _laid_out, _rows, _scratch, _tokens
from .lazytrain import (LT_ACT_GELU, LT_ACT_GELU_TANH, LT_ACT_RELU, LT_ACT_SILU, _check, _current,
                        _on, _stream_handle, lib)

_ACTIVATIONS = {"silu": LT_ACT_SILU, "gelu": LT_ACT_GELU, "gelu_tanh": LT_ACT_GELU_TANH,
                "relu": LT_ACT_RELU}


def _activation_code(name: str) -> int:
    code = _ACTIVATIONS.get(name)
    if code is None:
        raise ValueError(f"activation must be one of {', '.join(_ACTIVATIONS)}, got {name!r}")
    return code


def lt_int8_code_pitch(cols: int) -> int:
    """Bytes of a row of codes of a matrix with `cols` columns."""
    return -(-cols // 128) * 128


def _layout(codes: torch.Tensor, scales: torch.Tensor, rows: int, cols: int, device,
            what: str) -> Tuple[int, int]:
    """Addresses of a matrix's codes and scales."""
    pitch = lt_int8_code_pitch(cols)
    if codes.device != device or codes.dtype != torch.int8 or not codes.is_contiguous():
        raise ValueError(f"{what} must be contiguous int8 on {device}")
    if codes.numel() != rows * pitch:
        raise ValueError(f"{what} must have {rows} rows of {pitch} bytes")
    if scales.device != device or scales.dtype != torch.float32 or not scales.is_contiguous():
        raise ValueError(f"{what} scales must be contiguous float32 on {device}")
    if scales.numel() != rows:
        raise ValueError(f"{what} scales must be {rows}, one for each row")
    return codes.data_ptr(), scales.data_ptr()


def lt_int8_quantize(x: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor,
                     stream=None) -> None:
    """f10: quantizes x (rows, cols; float32 or bfloat16, contiguous rows) into codes (int8, rows of
    lt_int8_code_pitch(cols)) and a scale for each row."""
    stride = _rows(x, "x")
    rows, cols = x.shape
    code = _dtype_code(x, "x")
    device = x.device
    c, s = _layout(codes, scales, rows, cols, device, "codes")
    with _current(device):
        _check(lib().lt_int8_quantize(x.data_ptr(), code, rows, cols, stride, c, s,
                                      _stream_handle(stream, device)))
    increment_version([codes, scales])  # autograd's in-place rule


def lt_int8_matmul(a_codes: torch.Tensor, a_scales: torch.Tensor, b_codes: torch.Tensor,
                   b_scales: torch.Tensor, k: int, out: torch.Tensor,
                   workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """f11: out[i, j] = (sum over k of a_codes[i, k] * b_codes[j, k]) * a_scales[i] * b_scales[j] for
    operands that lt_int8_quantize made; out is (m, n), float32 or bfloat16, with contiguous
    rows."""
    stride = _rows(out, "out")
    m, n = out.shape
    code = _dtype_code(out, "out")
    device = out.device
    a, sa = _layout(a_codes, a_scales, m, k, device, "a_codes")
    b, sb = _layout(b_codes, b_scales, n, k, device, "b_codes")
    handle = _stream_handle(stream, device)
    held, ws, nbytes = _call_workspace(device, lib().lt_int8_matmul_workspace_bytes(m, n, k),
                                       workspace, stream)
    with _current(device):
        _check(lib().lt_int8_matmul(a, sa, b, sb, m, n, k, out.data_ptr(), code, stride, ws,
                                    nbytes, handle))
    increment_version([out])


class Int8Weight:
    """A linear layer's weight (out_features x in_features) in 8-bit integers with a scale for each
    output channel.  ``update`` quantizes the master weights into it again after a step."""

    __slots__ = ("rows", "cols", "codes", "scales")

    def __init__(self, rows: int, cols: int, codes: torch.Tensor, scales: torch.Tensor):
        self.rows, self.cols = int(rows), int(cols)
        _layout(codes, scales, self.rows, self.cols, codes.device, "codes")
        self.codes, self.scales = codes, scales

    @classmethod
    def empty(cls, rows: int, cols: int, device) -> "Int8Weight":
        return cls(rows, cols,
                   torch.empty(rows, lt_int8_code_pitch(cols), dtype=torch.int8, device=device),
                   torch.empty(rows, dtype=torch.float32, device=device))

    @classmethod
    def from_master(cls, w: torch.Tensor) -> "Int8Weight":
        """Quantizes a weight matrix (float32 or bfloat16) on the current stream."""
        if w.dim() != 2:
            raise ValueError(f"w must be a matrix (two dimensions, got {w.dim()})")
        weight = cls.empty(w.shape[0], w.shape[1], w.device)
        lt_int8_quantize(_laid_out(w, aligned=False), weight.codes, weight.scales)
        return weight

    def update(self, w: torch.Tensor, stream=None) -> None:
        if tuple(w.shape) != (self.rows, self.cols):
            raise ValueError(f"w must have shape {(self.rows, self.cols)}")
        with _on(stream, w.device):  # a copy of w belongs to the stream that reads it
            lt_int8_quantize(_laid_out(w, aligned=False), self.codes, self.scales)


def _call_workspace(device, need: int, workspace, stream=None):
    """What a call works in; an answer of 256 bytes stands for none."""
    if need <= 256 and workspace is None:
        return None, 0, 0
    return _scratch(device, need, workspace, stream)


def _input(x: torch.Tensor, weight: Int8Weight):
    t = _tokens(x, weight.cols, "x", aligned=False)
    if weight.codes.device != x.device:
        raise ValueError(f"the weight is on {weight.codes.device}, x on {x.device}")
    return t, _rows(t, "x"), _dtype_code(t, "x")


def int8_linear(x: torch.Tensor, weight: Int8Weight, out_dtype: torch.dtype = torch.bfloat16,
                workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """f11: x weight^T for x (..., in_features; float32 or bfloat16), each token quantized on the way.
    This and int8_gated_linear allocate and work on the current stream; for answering: nothing is
    kept for a backward pass."""
    t, stride, code = _input(x, weight)
    m, n, k, device = t.shape[0], weight.rows, weight.cols, x.device
    y = torch.empty(m, n, dtype=out_dtype, device=device)
    out = _dtype_code(y, "y")
    handle = _stream_handle(None, device)
    held, ws, nbytes = _call_workspace(device, lib().lt_int8_linear_workspace_bytes(m, n, k),
                                       workspace)
    with _current(device):
        _check(lib().lt_int8_linear(t.data_ptr(), code, stride, weight.codes.data_ptr(),
                                    weight.scales.data_ptr(), m, n, k, y.data_ptr(), out, n, ws,
                                    nbytes, handle))
    return y if x.dim() == 2 else y.view(*x.shape[:-1], n)


def int8_gated_linear(x: torch.Tensor, gate: Int8Weight, up: Int8Weight,
                      activation: str = "silu", out_dtype: torch.dtype = torch.bfloat16,
                      workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """f12: act(x gate^T) * (x up^T), the gated projections of a feed-forward block; activation is
    "silu", "gelu", "gelu_tanh" or "relu"."""
    t, stride, code = _input(x, gate)
    if (up.rows, up.cols) != (gate.rows, gate.cols):
        raise ValueError(f"up must have shape {(gate.rows, gate.cols)} as gate, got "
                         f"{(up.rows, up.cols)}")
    if up.codes.device != x.device:
        raise ValueError(f"the weight is on {up.codes.device}, x on {x.device}")
    act = _activation_code(activation)
    m, n, k, device = t.shape[0], gate.rows, gate.cols, x.device
    y = torch.empty(m, n, dtype=out_dtype, device=device)
    out = _dtype_code(y, "y")
    handle = _stream_handle(None, device)
    held, ws, nbytes = _call_workspace(device, lib().lt_int8_gated_workspace_bytes(m, n, k),
                                       workspace)
    with _current(device):
        _check(lib().lt_int8_gated(t.data_ptr(), code, stride, gate.codes.data_ptr(),
                                   gate.scales.data_ptr(), up.codes.data_ptr(),
                                   up.scales.data_ptr(), act, m, n, k, y.data_ptr(), out, n, ws,
                                   nbytes, handle))
    return y if x.dim() == 2 else y.view(*x.shape[:-1], n)
