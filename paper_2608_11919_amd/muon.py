"""Python binding of the matrix optimizer: Newton-Schulz orthogonalisation (f5) and the Muon
step with 8-bit momentum (f6); see include/lazytrain.h.  Argument marshalling only, in the
manner of the rest of the binding.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence

import torch

from . import lazytrain as _lt
from .lazytrain import (LT_DTYPE_BF16, LT_DTYPE_F32, LT_MAP_LINEAR, _List, _bf16_list, _check,
                        _check_block_size, _current, _device_of, _grad_code, _scalar, _state_ptr,
                        _stream_handle, _workspace, lib)

_DTYPES = {torch.float32: LT_DTYPE_F32, torch.bfloat16: LT_DTYPE_BF16}


def _sides(matrices, what):
    """Rows and columns of a list of matrices, as the library takes them (after lib())."""
    got = _lt._lists.sides(matrices)
    if got is not None:
        return got
    for i, m in enumerate(matrices):
        if m.dim() != 2:
            raise ValueError(f"{what}[{i}] must be a matrix (two dimensions, got {m.dim()})")
    n = len(matrices)
    return (bytes((ctypes.c_int64 * n)(*[m.shape[0] for m in matrices])),
            bytes((ctypes.c_int64 * n)(*[m.shape[1] for m in matrices])))


def _one_dtype(matrices, taken: _List, what) -> int:
    if taken.dtype in _DTYPES:
        return _DTYPES[taken.dtype]
    if not matrices:
        return LT_DTYPE_F32  # an empty list reads and writes nothing
    dt = matrices[0].dtype
    if dt not in _DTYPES or any(m.dtype != dt for m in matrices):
        raise TypeError(f"{what} must share one dtype, float32 or bfloat16")
    return _DTYPES[dt]


def lt_orthogonalize_workspace_bytes(rows: Sequence[int], cols: Sequence[int]) -> int:
    n = len(rows)
    return int(lib().lt_orthogonalize_workspace_bytes((ctypes.c_int64 * n)(*rows),
                                                      (ctypes.c_int64 * n)(*cols), n))


def lt_orthogonalize(matrices: Sequence[torch.Tensor], out: Sequence[torch.Tensor],
                     ns_steps: int = 5, workspace: Optional[torch.Tensor] = None,
                     stream=None) -> None:
    """f5: orthogonalises every matrix of a list into `out` (contiguous matrices of the same
    shapes; each list float32 or bfloat16)."""
    if len(matrices) != len(out):
        raise ValueError("tensor lists must be of equal length")
    device = _device_of(matrices)
    src = _List(matrices, device, what="matrices")
    dst = _List(out, device, what="out")
    rows, cols = _sides(matrices, "matrices")
    if _sides(out, "out") != (rows, cols):
        for i, (o, m) in enumerate(zip(out, matrices)):
            if o.shape != m.shape:
                raise ValueError(f"out[{i}] must have shape {tuple(m.shape)}")
    n = len(matrices)
    nbytes = int(lib().lt_orthogonalize_workspace_bytes(rows, cols, n))
    ws = _workspace(device, nbytes, workspace, stream, "orthogonalize")
    with _current(device):
        _check(lib().lt_orthogonalize(
            src.ptrs, _one_dtype(matrices, src, "matrices"), dst.ptrs,
            _one_dtype(out, dst, "out"), rows, cols, n, int(ns_steps), ws.data_ptr(),
            ws.numel() * ws.element_size(), _stream_handle(stream, device)))


def lt_muon_workspace_bytes(rows: Sequence[int], cols: Sequence[int], block_size: int) -> int:
    n = len(rows)
    return int(lib().lt_muon_workspace_bytes((ctypes.c_int64 * n)(*rows),
                                             (ctypes.c_int64 * n)(*cols), n, int(block_size)))


def lt_muon_step(params: Sequence[torch.Tensor], grads: Sequence[torch.Tensor],
                 m_codes: Sequence[torch.Tensor], m_absmax: Sequence[torch.Tensor],
                 block_size: int, lr: float, momentum: float = 0.95, weight_decay: float = 0.0,
                 ns_steps: int = 5, nesterov: bool = True, update_rms: float = 0.2,
                 coef: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
                 workspace: Optional[torch.Tensor] = None, stream=None, params_bf16=None,
                 code_map: int = LT_MAP_LINEAR,
                 step_state: Optional[torch.Tensor] = None) -> None:
    """f6: one Muon step in place on params (float32 matrices), codes and absmax (see
    include/lazytrain.h); grads have the parameters' sizes, in float32 or bfloat16;
    params_bf16, coef, status and step_state as in lt_hybrid8bit_adamw_step."""
    n = len(params)
    if not (len(grads) == len(m_codes) == len(m_absmax) == n):
        raise ValueError("tensor lists must be of equal length")
    device = _device_of(params, coef, status)
    p = _List(params, device, torch.float32, "params")
    g = _List(grads, device, what="grads")
    mq = _List(m_codes, device, torch.int8, "m_codes")
    ma = _List(m_absmax, device, torch.float32, "m_absmax")
    gdt = _grad_code(grads, g)
    _check_block_size(block_size)
    rows, cols = _sides(params, "params")
    if _lt._lists.sides(grads) != (rows, cols):
        for i in range(n):  # a gradient may be flat, but no matrix of another shape
            if grads[i].dim() != 1 and grads[i].shape != params[i].shape:
                raise ValueError(f"grads[{i}] must have shape {tuple(params[i].shape)}")
    if not (g.numels == p.numels == mq.numels and
            _lt._lists.covers(p.numels, ma.numels, int(block_size))):
        for i in range(n):
            size = params[i].numel()
            nb = -(-size // int(block_size))
            if grads[i].numel() != size or m_codes[i].numel() != size:
                raise ValueError(f"tensor {i}: params, grads and codes must have {size} elements")
            if m_absmax[i].numel() < nb:
                raise ValueError(f"tensor {i}: m_absmax needs {nb} entries")
    wb = _bf16_list(params_bf16, params, device, p.numels)
    nbytes = int(lib().lt_muon_workspace_bytes(rows, cols, n, int(block_size)))
    ws = _workspace(device, nbytes, workspace, stream, "muon")
    with _current(device):
        _check(lib().lt_muon_step(
            p.ptrs, g.ptrs, gdt, mq.ptrs, ma.ptrs, wb, rows, cols, n, int(block_size),
            int(code_map), float(lr), float(momentum), int(bool(nesterov)), float(weight_decay),
            float(update_rms), int(ns_steps), _scalar(coef, device, torch.float32, "coef"),
            _scalar(status, device, torch.int32, "status"), _state_ptr(step_state, device),
            ws.data_ptr(), ws.numel() * ws.element_size(), _stream_handle(stream, device)))
