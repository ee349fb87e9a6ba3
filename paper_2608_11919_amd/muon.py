"""Python binding of the matrix optimizer: Newton-Schulz orthogonalisation (f5) and the Muon
step with 8-bit momentum (f6); see include/lazytrain.h.  Argument marshalling only, in the
manner of the rest of the binding.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence

import torch

from . import lazytrain as _lt
from .lazytrain import (LT_DTYPE_BF16, LT_DTYPE_F32, LT_ERR_WORKSPACE, LT_MAP_LINEAR,
                        Hybrid8bitAdamW, _List, _bf16_list, _check, _check_block_size, _current,
                        _device_of, _grad_code, _list_workspace, _scalar, _state_ptr,
                        _stream_handle, lib)

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
    handle = _stream_handle(stream, device)
    ws = _list_workspace(device, nbytes, workspace, stream, "orthogonalize", handle)
    with _current(device):
        _check(lib().lt_orthogonalize(
            src.ptrs, _one_dtype(matrices, src, "matrices"), dst.ptrs,
            _one_dtype(out, dst, "out"), rows, cols, n, int(ns_steps), ws.data_ptr(),
            ws.numel() * ws.element_size(), handle))


def lt_muon_workspace_bytes(rows: Sequence[int], cols: Sequence[int], block_size: int) -> int:
    n = len(rows)
    return int(lib().lt_muon_workspace_bytes((ctypes.c_int64 * n)(*rows),
                                             (ctypes.c_int64 * n)(*cols), n, int(block_size)))


class _MuonCall:
    """A Muon step's arguments, checked as far as the binding does, with its workspace: run()
    enqueues it, check() has the library refuse what it would, and enqueues nothing."""

    __slots__ = ("device", "args", "workspace", "handle", "held")

    def __init__(self, params, grads, m_codes, m_absmax, block_size, lr, momentum=0.95,
                 weight_decay=0.0, ns_steps=5, nesterov=True, update_rms=0.2, coef=None,
                 status=None, workspace=None, stream=None, params_bf16=None,
                 code_map=LT_MAP_LINEAR, step_state=None):
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
                    raise ValueError(f"tensor {i}: params, grads and codes must have {size} "
                                     "elements")
                if m_absmax[i].numel() < nb:
                    raise ValueError(f"tensor {i}: m_absmax needs {nb} entries")
        wb = _bf16_list(params_bf16, params, device, p.numels)
        nbytes = int(lib().lt_muon_workspace_bytes(rows, cols, n, int(block_size)))
        self.device, self.handle = device, _stream_handle(stream, device)
        self.workspace = _list_workspace(device, nbytes, workspace, stream, "muon", self.handle)
        self.args = (p.ptrs, g.ptrs, gdt, mq.ptrs, ma.ptrs, wb, rows, cols, n, int(block_size),
                     int(code_map), float(lr), float(momentum), int(bool(nesterov)),
                     float(weight_decay), float(update_rms), int(ns_steps),
                     _scalar(coef, device, torch.float32, "coef"),
                     _scalar(status, device, torch.int32, "status"),
                     _state_ptr(step_state, device))
        self.held = (params, grads, m_codes, m_absmax, params_bf16, coef, status, step_state)

    def check(self) -> None:
        with _current(self.device):
            rc = lib().lt_muon_step(*self.args, 0, 0, self.handle)
        if rc != LT_ERR_WORKSPACE:  # what it looks at last
            _check(rc)

    def run(self) -> None:
        ws = self.workspace
        with _current(self.device):
            _check(lib().lt_muon_step(*self.args, ws.data_ptr(), ws.numel() * ws.element_size(),
                                      self.handle))


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
    _MuonCall(params, grads, m_codes, m_absmax, block_size, lr, momentum, weight_decay, ns_steps,
              nesterov, update_rms, coef, status, workspace, stream, params_bf16, code_map,
              step_state).run()


# ------------------------------------------------------------- optimizer object

class HybridMuon(Hybrid8bitAdamW):
    """Muon for matrices, 8-bit AdamW for the rest, under one global norm: a step is
    lt_grad_sqnorm -> lt_clip_coef -> the AdamW steps -> lt_muon_step, on one stream without a
    host synchronization, with the step count, the skips and the checkpoints of
    Hybrid8bitAdamW.

    ``matrices`` says which parameters Muon updates, one truth value each; by default every
    parameter of two dimensions with two rows and two columns or more.  Embeddings and output
    heads are commonly left to AdamW.  A Muon update has a root mean square of about
    ``update_rms`` times lr, 0.2 being about AdamW's, so that one learning rate serves both.
    Its momentum is held in 8 bits in blocks of ``block_size`` with ``muon_code_map``'s codes
    (linear: nothing divides by it, so small values may round to 0)."""

    def __init__(self, params: Sequence[torch.Tensor], lr: float = 1e-5, momentum: float = 0.95,
                 nesterov: bool = True, ns_steps: int = 5, update_rms: float = 0.2,
                 matrices: Optional[Sequence[bool]] = None, muon_code_map: int = LT_MAP_LINEAR,
                 **adamw):
        params = list(params)
        if matrices is None:
            matrices = [p.dim() == 2 and min(p.shape) > 1 for p in params]
        matrices = [bool(m) for m in matrices]
        if len(matrices) != len(params):
            raise ValueError("matrices needs one truth value per parameter")
        for i, (m, p) in enumerate(zip(matrices, params)):
            if m and (p.dim() != 2 or not p.is_contiguous()):
                raise ValueError(f"parameter {i} must be a contiguous matrix")
        self.is_matrix = matrices
        self.idx_muon = [i for i, m in enumerate(matrices) if m]
        self.momentum, self.nesterov, self.ns_steps = momentum, nesterov, ns_steps
        self.update_rms, self.muon_code_map = update_rms, muon_code_map
        super().__init__(params, lr=lr, **adamw)
        dev = self.device
        mine = [self.params[i] for i in self.idx_muon]
        self.muon_codes = [torch.zeros(p.numel(), dtype=torch.int8, device=dev) for p in mine]
        self.muon_absmax = [torch.zeros(-(-p.numel() // self.block_size), dtype=torch.float32,
                                        device=dev) for p in mine]
        torch.cuda.synchronize(dev)  # steps may come on any stream

    def _elsewhere(self) -> frozenset:
        return frozenset(self.idx_muon)

    def _prepare_elsewhere(self, grads, stream):
        if not self.idx_muon:
            return None
        wb = self.params_bf16
        call = _MuonCall(
            [self.params[i] for i in self.idx_muon], [grads[i] for i in self.idx_muon],
            self.muon_codes, self.muon_absmax, self.block_size, lr=self.lr,
            momentum=self.momentum, weight_decay=self.weight_decay, ns_steps=self.ns_steps,
            nesterov=self.nesterov, update_rms=self.update_rms, coef=self.coef,
            status=self.status, stream=stream,
            params_bf16=None if wb is None else [wb[i] for i in self.idx_muon],
            code_map=self.muon_code_map, step_state=self._state)
        call.check()
        return call

    def _step_elsewhere(self, prepared) -> None:
        if prepared is not None:
            prepared.run()

    def state_dict(self, stream=None) -> dict:
        state = super().state_dict(stream)
        host = lambda ts: [t.detach().cpu().clone() for t in ts]
        state["muon"] = {"is_matrix": list(self.is_matrix), "momentum": self.momentum,
                         "nesterov": self.nesterov, "ns_steps": self.ns_steps,
                         "update_rms": self.update_rms, "code_map": self.muon_code_map,
                         "codes": host(self.muon_codes), "absmax": host(self.muon_absmax)}
        return state

    def load_state_dict(self, state: dict) -> None:
        mine = state.get("muon")
        if mine is None or list(mine["is_matrix"]) != list(self.is_matrix):
            raise ValueError("the checkpoint's Muon matrices differ from this optimizer's")
        if mine["code_map"] != self.muon_code_map:
            raise ValueError("the checkpoint's code map of the momentum differs")
        for name, tensors in (("codes", self.muon_codes), ("absmax", self.muon_absmax)):
            if [t.shape for t in mine[name]] != [t.shape for t in tensors]:
                raise ValueError(f"muon {name}: shapes differ from the checkpoint")
        super().load_state_dict(state)
        self.momentum, self.nesterov = mine["momentum"], mine["nesterov"]
        self.ns_steps, self.update_rms = mine["ns_steps"], mine["update_rms"]
        for name, tensors in (("codes", self.muon_codes), ("absmax", self.muon_absmax)):
            for a, b in zip(tensors, mine[name]):
                a.copy_(b)
        torch.cuda.synchronize(self.device)
