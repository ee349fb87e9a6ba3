"""The gated projections of a feed-forward block in bfloat16 (f13 and f14; see include/lazytrain.h):
act(x gate^T) * (x up^T) with the weights the optimizer keeps in bfloat16, for answering and for
training, with the gradients of the tokens and of both weights.
"""
from __future__ import annotations

import threading
import weakref
from typing import Optional, Tuple

import torch
from torch.autograd import forward_ad

from .fp8 import _dtype_code, _laid_out, _rows, _scratch, _tokens
from .int8 import _activation_code, _call_workspace
from .lazytrain import _capturing, _check, _current, _stream_handle, lib


def _weights(gate: torch.Tensor, up: torch.Tensor, device):
    """The weights as the library takes them, and their row strides."""
    if gate.dim() != 2 or up.shape != gate.shape:
        raise ValueError(f"gate and up must be matrices of one shape, got {tuple(gate.shape)} and "
                         f"{tuple(up.shape)}")
    return (*_weight(gate, "gate", device), *_weight(up, "up", device))


def _weight(w: torch.Tensor, what: str, device):
    if w.dtype != torch.bfloat16:
        raise TypeError(f"{what} must be bfloat16, got {w.dtype}")
    if w.device != device:
        raise ValueError(f"{what} is on {w.device}, not on {device}")
    if w.is_contiguous() and not w.data_ptr() % 16:
        return w, w.shape[1]
    w = _laid_out(w)
    return w, _rows(w, what)


def _input(x: torch.Tensor, features: int) -> Tuple[torch.Tensor, int]:
    if x.dtype != torch.bfloat16:
        raise TypeError(f"x must be bfloat16, got {x.dtype}")
    if x.dim() == 2 and x.shape[1] == features and x.is_contiguous() and not x.data_ptr() % 16:
        return x, features
    t = _tokens(x, features, "x")
    return t, _rows(t, "x")


def _forward(x, gate, up, activation, out_dtype, keep, workspace):
    act = _activation_code(activation)
    g, g_stride, u, u_stride = _weights(gate, up, x.device)
    n, k = g.shape
    t, x_stride = _input(x, k)
    m, device = t.shape[0], x.device
    h = torch.empty(m, n, dtype=out_dtype, device=device)
    out = _dtype_code(h, "out")
    saved = None
    if keep:
        saved = torch.empty(6 * m * (-(-n // 8) * 8), dtype=torch.uint8, device=device)
    ws, nbytes, handle = 0, 0, _stream_handle(None, device)
    strides = x_stride | g_stride | u_stride
    copies = k % 64 or strides % 8 or strides >= 1 << 22
    if workspace is not None or m > 16 or (k > 4096 and not copies):
        need = int(lib().lt_gated_forward_workspace_bytes(m, n, k, x_stride, g_stride, u_stride))
        held, ws, nbytes = _call_workspace(device, need, workspace)
    with _current(device):
        _check(lib().lt_gated_forward(t.data_ptr(), x_stride, g.data_ptr(), g_stride, u.data_ptr(),
                                      u_stride, act, m, n, k, h.data_ptr(), out, n,
                                      saved.data_ptr() if keep else 0, ws, nbytes, handle))
    return h if x.dim() == 2 else h.view(*x.shape[:-1], n), saved


def gated_linear(x: torch.Tensor, gate: torch.Tensor, up: torch.Tensor, activation: str = "silu",
                 out_dtype: torch.dtype = torch.bfloat16,
                 workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """f13: act(x gate^T) * (x up^T) for x (..., in_features) and two weights (out_features x
    in_features), all bfloat16; activation is "silu", "gelu", "gelu_tanh" or "relu".  For answering:
    nothing is kept for a backward pass.  This and the functions below allocate and work on the
    current stream."""
    return _forward(x, gate, up, activation, out_dtype, False, workspace)[0]


def gated_linear_forward(x: torch.Tensor, gate: torch.Tensor, up: torch.Tensor,
                         activation: str = "silu", out_dtype: torch.dtype = torch.bfloat16):
    """As gated_linear, and what the backward pass needs of its results: six bytes for each, in one
    tensor of bytes."""
    return _forward(x, gate, up, activation, out_dtype, True, None)


def gated_linear_backward(dh: torch.Tensor, saved: torch.Tensor, x: torch.Tensor,
                          gate: torch.Tensor, up: torch.Tensor,
                          out_dtype: torch.dtype = torch.bfloat16,
                          grad_dtype: torch.dtype = torch.bfloat16):
    """(dx, dgate, dup) of gated_linear_forward: dx in out_dtype with x's shape, the weights'
    gradients in grad_dtype (float32 leaves out their last rounding; the products' operands are
    bfloat16 all the same).  dh is float32 or bfloat16."""
    return _backward(dh, saved, x, gate, up, tuple(x.shape[:-1]), tuple(gate.shape), out_dtype,
                     grad_dtype, True, True)


def _backward(dh, saved, x, gate, up, leading, shape, out_dtype, grad_dtype, want_dx, want_dw):
    """dx needs the weights, the weights' gradients x; what is not needed may be None."""
    n, k = shape
    device = dh.device
    d_code = _dtype_code(dh, "dh")
    if dh.dim() == 2 and dh.shape[1] == n and dh.is_contiguous():
        d, d_stride = dh, n
    else:
        d = _tokens(dh, n, "dh", aligned=False)
        d_stride = _rows(d, "dh")
    m = d.shape[0]
    if tuple(dh.shape[:-1]) != leading:
        raise ValueError(f"dh must have shape {leading + (n,)}, got {tuple(dh.shape)}")
    if (saved.device != device or saved.dtype != torch.uint8 or not saved.is_contiguous() or
            saved.numel() != 6 * m * (-(-n // 8) * 8)):
        raise ValueError("saved must be what gated_linear_forward kept of these tokens")
    x_at = g_at = u_at = dx_at = dgate_at = dup_at = dx_code = grad_code = 0
    x_stride = g_stride = u_stride = k
    dx = dgate = dup = None
    if want_dx:
        g, g_stride, u, u_stride = _weights(gate, up, device)
        dx = torch.empty(m, k, dtype=out_dtype, device=device)
        dx_code = _dtype_code(dx, "dx")
        g_at, u_at, dx_at = g.data_ptr(), u.data_ptr(), dx.data_ptr()
    if want_dw:
        if x.device != device:
            raise ValueError(f"x is on {x.device}, dh on {device}")
        t, x_stride = _input(x, k)
        if t.shape[0] != m:
            raise ValueError(f"x has {t.shape[0]} tokens, dh {m}")
        dgate = torch.empty(n, k, dtype=grad_dtype, device=device)
        dup = torch.empty(n, k, dtype=grad_dtype, device=device)
        grad_code = _dtype_code(dgate, "the weights' gradients")
        x_at, dgate_at, dup_at = t.data_ptr(), dgate.data_ptr(), dup.data_ptr()
    if not want_dx and not want_dw:
        return None, None, None
    handle = _stream_handle(None, device)
    need = lib().lt_gated_backward_workspace_bytes(m, n, k, x_stride, g_stride, u_stride, want_dx,
                                                   want_dw)
    held, ws, nbytes = _scratch(device, need, None, None)
    with _current(device):
        _check(lib().lt_gated_backward(d.data_ptr(), d_code, d_stride, saved.data_ptr(), x_at,
                                       x_stride, g_at, g_stride, u_at, u_stride, m, n, k, dx_at,
                                       dx_code, k, dgate_at, k, dup_at, k, grad_code, ws, nbytes,
                                       handle))
    if dx is not None and len(leading) != 1:
        dx = dx.view(*leading, k)
    return dx, dgate, dup


# Graphs of GatedLinear that were made on the default stream, as weak references without callbacks:
# threads add to them while another looks, which a WeakSet's iteration does not bear.
_on_default = []
_on_default_lock = threading.Lock()
_on_default_most = 256  # from here on those that are gone are dropped


def _made_on_default(ctx) -> None:
    global _on_default, _on_default_most
    with _on_default_lock:
        if len(_on_default) >= _on_default_most:
            _on_default = [r for r in _on_default if r() is not None]
            _on_default_most = 2 * len(_on_default) + 256
        _on_default.append(weakref.ref(ctx))


def _held_on_default(leaves) -> bool:
    """Whether one of these graphs lives and holds a leaf of `leaves`, a set of ids."""
    with _on_default_lock:
        graphs = list(_on_default)
    return any(c is not None and not leaves.isdisjoint(c.leaves) for c in (r() for r in graphs))


class GatedLinear(torch.autograd.Function):
    """``GatedLinear.apply(x, gate, up, activation)``: gated_linear with gradients for x, gate and up
    (for instance the optimizer's bf16 copies).  The backward pass reads x and the weights again:
    one of them changed in place meanwhile raises, like autograd's own.  First derivatives only: a
    backward pass that is itself to be differentiated raises, and so does a tangent of forward mode.
    Where gradients are off it is gated_linear and keeps nothing; the result has the same bits.

    Autograd adds up a leaf's gradient on the stream that its first graph was made on, for as long
    as a graph of the leaf lives.  Under capture that cannot be the default stream (the process would
    end with the capture): a captured call is refused while the graph of an earlier call, made there,
    holds one of its leaves."""

    @classmethod
    def apply(cls, x, gate, up, activation="silu"):
        # gradients off, which forward below cannot see: it would keep its results.  A tangent of
        # forward mode would get lost; autograd refuses it
        if not torch.is_grad_enabled() and not any(
                forward_ad.unpack_dual(t).tangent is not None for t in (x, gate, up)):
            return gated_linear(x, gate, up, activation)
        return super().apply(x, gate, up, activation)

    @staticmethod
    def forward(ctx, x, gate, up, activation="silu"):
        want_dx, want_dw = ctx.needs_input_grad[0], any(ctx.needs_input_grad[1:3])
        if x.is_cuda and (want_dx or want_dw):
            # a graph holds its leaves: their ids stay theirs as long as it lives
            leaves = {id(t) for t in (x, gate, up) if t.requires_grad and t.is_leaf}
            if _stream_handle(None, x.device) == 0:
                ctx.leaves = leaves
                _made_on_default(ctx)
            elif _capturing(None, x.device) and _held_on_default(leaves):
                raise RuntimeError("GatedLinear is being captured while a graph made on the default "
                                   "stream holds the same leaf: let go of that graph's results "
                                   "first, or make it on another stream")
        h, saved = _forward(x, gate, up, activation, torch.bfloat16, want_dx or want_dw, None)
        ctx.save_for_backward(saved, x if want_dw else None, *((gate, up) if want_dx
                                                               else (None, None)))
        ctx.leading, ctx.shape = tuple(x.shape[:-1]), tuple(gate.shape)
        return h

    @staticmethod
    def backward(ctx, dh):
        if torch.is_grad_enabled() and (dh.requires_grad or any(ctx.needs_input_grad[:3])):
            raise RuntimeError("GatedLinear has first derivatives only: its backward pass cannot be "
                               "part of a graph (create_graph=True)")
        saved, x, gate, up = ctx.saved_tensors
        need = ctx.needs_input_grad
        dx, dgate, dup = _backward(dh, saved, x, gate, up, ctx.leading, ctx.shape, torch.bfloat16,
                                   torch.bfloat16, need[0], need[1] or need[2])
        return dx, dgate if need[1] else None, dup if need[2] else None, None
