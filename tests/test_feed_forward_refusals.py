"""The feed-forward operators' refusals that need no GPU: arrays that overlap, strides, sizes, types
and addresses that no launch could take.  Addresses are made up; every call here returns before
it looks at one."""
import pytest
import torch

import paper_2608_11919_amd as lt
from paper_2608_11919_amd.lazytrain import lib

BASE = 1 << 40  # an address on every boundary, which nothing reads
WS = 100 * BASE


def quantize(x=BASE, dtype=lt.LT_DTYPE_BF16, rows=300, cols=200, stride=200, codes=2 * BASE,
             scales=3 * BASE):
    return lib().lt_int8_quantize(x, dtype, rows, cols, stride, codes, scales, None)


def matmul(a=BASE, a_scales=2 * BASE, b=3 * BASE, b_scales=4 * BASE, m=40, n=48, k=130,
           out=5 * BASE, dtype=lt.LT_DTYPE_F32, stride=48, ws=WS, ws_bytes=1 << 30):
    return lib().lt_int8_matmul(a, a_scales, b, b_scales, m, n, k, out, dtype, stride, ws, ws_bytes,
                                None)


def linear(x=BASE, dtype=lt.LT_DTYPE_F32, x_stride=130, w=2 * BASE, w_scales=3 * BASE, m=4, n=48,
           k=130, out=4 * BASE, out_dtype=lt.LT_DTYPE_F32, stride=48, ws=WS, ws_bytes=1 << 30):
    return lib().lt_int8_linear(x, dtype, x_stride, w, w_scales, m, n, k, out, out_dtype, stride,
                                ws, ws_bytes, None)


def int8_gated(x=BASE, dtype=lt.LT_DTYPE_F32, x_stride=130, gate=2 * BASE, gs=3 * BASE,
               up=4 * BASE, us=5 * BASE, act=0, m=4, n=48, k=130, out=6 * BASE,
               out_dtype=lt.LT_DTYPE_F32, stride=48, ws=WS, ws_bytes=1 << 30):
    return lib().lt_int8_gated(x, dtype, x_stride, gate, gs, up, us, act, m, n, k, out, out_dtype,
                               stride, ws, ws_bytes, None)


def forward(x=BASE, xs=130, gate=2 * BASE, gs=130, up=3 * BASE, us=130, act=0, m=40, n=48, k=130,
            out=4 * BASE, dtype=lt.LT_DTYPE_BF16, stride=48, saved=5 * BASE, ws=WS,
            ws_bytes=1 << 30):
    return lib().lt_gated_forward(x, xs, gate, gs, up, us, act, m, n, k, out, dtype, stride, saved,
                                  ws, ws_bytes, None)


def backward(dh=BASE, dh_dtype=lt.LT_DTYPE_BF16, dhs=48, saved=2 * BASE, x=3 * BASE, xs=130,
             gate=4 * BASE, gs=130, up=5 * BASE, us=130, m=40, n=48, k=130, dx=6 * BASE,
             dx_dtype=lt.LT_DTYPE_BF16, dxs=130, dgate=7 * BASE, dgs=130, dup=8 * BASE, dus=130,
             grad_dtype=lt.LT_DTYPE_BF16, ws=WS, ws_bytes=1 << 30):
    return lib().lt_gated_backward(dh, dh_dtype, dhs, saved, x, xs, gate, gs, up, us, m, n, k, dx,
                                   dx_dtype, dxs, dgate, dgs, dup, dus, grad_dtype, ws, ws_bytes,
                                   None)


@pytest.mark.parametrize("call", [
    lambda: quantize(codes=BASE + (300 * 200 * 2 - 1) // 16 * 16),
    lambda: quantize(x=2 * BASE + 300 * 256 - 2),
    lambda: quantize(scales=2 * BASE + 300 * 256 - 4),
    lambda: quantize(scales=BASE + 4),
    lambda: matmul(out=BASE + 40 * 256 - 16),
    lambda: matmul(out=3 * BASE + 48 * 256 - 16),
    lambda: matmul(a_scales=5 * BASE),
    lambda: matmul(b_scales=5 * BASE + 64),
    lambda: matmul(k=12800, out=WS),
    lambda: matmul(k=12800, ws=BASE),
    lambda: linear(out=BASE + ((3 * 130 + 130) * 4 - 1) // 16 * 16),
    lambda: linear(out=2 * BASE),
    lambda: linear(w_scales=4 * BASE),
    lambda: linear(m=40, ws=2 * BASE),
    lambda: linear(m=40, out=WS),
    lambda: int8_gated(out=4 * BASE),
    lambda: int8_gated(us=6 * BASE),
    lambda: int8_gated(m=40, ws=4 * BASE),
    lambda: forward(out=BASE),
    lambda: forward(out=3 * BASE + 47 * 130 * 2 // 16 * 16),
    lambda: forward(saved=2 * BASE + 64),
    lambda: forward(saved=4 * BASE + 64),
    lambda: forward(ws=5 * BASE),
    lambda: forward(ws=BASE),
    lambda: backward(dx=BASE),
    lambda: backward(dx=4 * BASE),
    lambda: backward(dgate=3 * BASE),
    lambda: backward(dup=7 * BASE + 16),
    lambda: backward(ws=2 * BASE),
    lambda: backward(dup=WS),
])
def test_overlaps(call):
    assert call() == lt.LT_ERR_INVALID_ARG
    assert b"overlap" in lib().lt_last_error()


BIG = 1 << 21


@pytest.mark.parametrize("call", [
    lambda: quantize(stride=199),
    lambda: quantize(stride=1 << 62),
    lambda: quantize(rows=1 << 31, cols=1, stride=1),
    lambda: quantize(rows=-1),
    lambda: quantize(dtype=2),
    lambda: quantize(x=0),
    lambda: quantize(scales=0),
    lambda: matmul(stride=47),
    lambda: matmul(stride=1 << 60),
    lambda: matmul(m=1 << 28),
    lambda: matmul(m=1 << 20, n=1 << 20, stride=1 << 20),
    lambda: matmul(k=(1 << 17) + 1),
    lambda: matmul(k=-1),
    lambda: matmul(dtype=7),
    lambda: matmul(a=0),
    lambda: linear(x_stride=129),
    lambda: linear(x_stride=1 << 61),
    lambda: linear(n=1 << 28, stride=1 << 28),
    lambda: linear(k=(1 << 17) + 1, x_stride=1 << 18),
    lambda: linear(dtype=5),
    lambda: linear(out_dtype=5),
    lambda: linear(w=0),
    lambda: int8_gated(act=4),
    lambda: int8_gated(act=-1),
    lambda: int8_gated(up=0),
    lambda: int8_gated(us=0),
    lambda: int8_gated(stride=47),
    lambda: forward(xs=129),
    lambda: forward(gs=129),
    lambda: forward(us=1 << 60),
    lambda: forward(stride=47),
    lambda: forward(m=BIG),
    lambda: forward(n=BIG, stride=BIG),
    lambda: forward(k=BIG, xs=BIG, gs=BIG, us=BIG),
    lambda: forward(m=BIG - 1, n=BIG - 1, stride=BIG),
    lambda: forward(act=4),
    lambda: forward(dtype=3),
    lambda: forward(up=0),
    lambda: forward(out=0),
    lambda: backward(dhs=47),
    lambda: backward(dxs=129),
    lambda: backward(dgs=129),
    lambda: backward(dgate=0),
    lambda: backward(dup=0),
    lambda: backward(x=0),
    lambda: backward(gate=0),
    lambda: backward(saved=0),
    lambda: backward(dh_dtype=3),
    lambda: backward(grad_dtype=3),
    lambda: backward(m=-1),
    lambda: backward(k=BIG, xs=BIG, gs=BIG, us=BIG, dxs=BIG, dgs=BIG, dus=BIG),
])
def test_arguments(call):
    assert call() == lt.LT_ERR_INVALID_ARG


@pytest.mark.parametrize("call", [
    lambda: quantize(x=BASE + 1),
    lambda: quantize(codes=BASE * 2 + 8),
    lambda: matmul(a=BASE + 4),
    lambda: matmul(out=5 * BASE + 4),
    lambda: matmul(b_scales=4 * BASE + 2),
    lambda: linear(x=BASE + 2),
    lambda: linear(w=2 * BASE + 8),
    lambda: int8_gated(up=4 * BASE + 8),
    lambda: forward(x=BASE + 2),
    lambda: forward(gate=2 * BASE + 8),
    lambda: forward(saved=5 * BASE + 8),
    lambda: backward(dh=BASE + 1),
    lambda: backward(saved=2 * BASE + 8),
    lambda: backward(dx=6 * BASE + 2),
    lambda: backward(x=3 * BASE + 2),
    lambda: backward(up=5 * BASE + 8),
])
def test_alignment(call):
    assert call() == lt.LT_ERR_ALIGNMENT


@pytest.mark.parametrize("call", [
    lambda: matmul(k=12800, ws=0),
    lambda: matmul(k=12800, ws_bytes=256),
    lambda: linear(m=40, ws=0),
    lambda: linear(m=40, ws=WS + 64),
    lambda: int8_gated(m=40, ws_bytes=100),
    lambda: forward(ws=0),
    lambda: forward(ws_bytes=1000),
    lambda: backward(ws=0),
    lambda: backward(ws_bytes=1000),
])
def test_workspaces(call):
    assert call() == lt.LT_ERR_WORKSPACE


def test_nothing_to_do():
    """Empty results are fine without a device and without arrays."""
    assert quantize(rows=0, x=0, codes=0, scales=0) == lt.LT_OK
    assert matmul(m=0, out=0, a=0, a_scales=0) == lt.LT_OK
    assert linear(n=0, out=0, w=0, w_scales=0) == lt.LT_OK
    assert int8_gated(m=0, x=0, out=0) == lt.LT_OK
    assert forward(m=0, x=0, out=0, saved=0) == lt.LT_OK
    assert backward(dx=0, dgate=0, dup=0) == lt.LT_OK
    assert backward(k=0, xs=0, gs=0, us=0) == lt.LT_OK


def test_sizes_of_memory():
    L = lib()
    assert [lt.lt_int8_code_pitch(c) for c in (0, 1, 128, 129)] == [0, 128, 128, 256]
    assert [L.lt_int8_code_pitch(c) for c in (-1, 0, 1, 128, 129)] == [0, 0, 128, 128, 256]
    assert L.lt_int8_matmul_workspace_bytes(4, 4, 4) == 256
    assert L.lt_int8_matmul_workspace_bytes(40, 48, 1 << 18) == 0
    assert L.lt_int8_linear_workspace_bytes(100, 4, 300) >= 100 * 384 + 400
    assert L.lt_int8_linear_workspace_bytes(4, 4, 8192) == 256
    assert L.lt_int8_linear_workspace_bytes(16, 4, 2048) == 256
    assert L.lt_int8_linear_workspace_bytes(16, 4, 2049) > 16 * 2049
    assert L.lt_int8_linear_workspace_bytes(1, 4, 8193) > 8193
    assert L.lt_int8_gated_workspace_bytes(-1, 4, 300) == 0
    for m, n, k in ((40, 0, 500), (0, 40, 500), (40, 40, 0), (0, 0, 0)):
        assert L.lt_int8_matmul_workspace_bytes(m, n, k) == 256
        assert L.lt_int8_linear_workspace_bytes(m, n, k) >= 256
        assert L.lt_int8_gated_workspace_bytes(m, n, k) >= 256
        assert L.lt_gated_forward_workspace_bytes(m, n, k, 9, 9, 9) >= 256
        assert L.lt_gated_backward_workspace_bytes(m, n, k, k, k, k, 1, 1) >= 256
    assert L.lt_gated_saved_bytes(3, 9) == 6 * 3 * 16
    assert L.lt_gated_saved_bytes(3, 1 << 21) == 0
    assert L.lt_gated_forward_workspace_bytes(64, 64, 64, 64, 64, 64) == 256
    assert L.lt_gated_forward_workspace_bytes(64, 32, 64, 65, 64, 64) == 64 * 128
    assert L.lt_gated_backward_workspace_bytes(-1, 1, 1, 1, 1, 1, 1, 1) == 0
    slopes, tail = 128 * 512 * 2, 64 * 304 * 2
    for want, bytes_ in (((0, 0), slopes), ((1, 0), slopes + 2 * tail), ((0, 1), slopes + tail)):
        assert L.lt_gated_backward_workspace_bytes(100, 200, 304, 304, 304, 304, *want) == bytes_
    # columns that are no multiple of 8: whole copies
    assert L.lt_gated_backward_workspace_bytes(100, 200, 300, 300, 300, 300, 1, 1) == \
        slopes + 2 * 256 * 320 * 2 + 128 * 320 * 2


def test_tensors():
    """What the binding refuses before the library is called."""
    f = lambda *s, dtype=torch.bfloat16: torch.zeros(*s, dtype=dtype)
    with pytest.raises(ValueError, match="activation"):
        lt.gated_linear(f(4, 8), f(6, 8), f(6, 8), "swish")
    with pytest.raises(TypeError, match="x must be bfloat16"):
        lt.gated_linear(f(4, 8, dtype=torch.float32), f(6, 8), f(6, 8))
    with pytest.raises(TypeError, match="up must be bfloat16"):
        lt.gated_linear(f(4, 8), f(6, 8), f(6, 8, dtype=torch.float32))
    with pytest.raises(ValueError, match="one shape"):
        lt.gated_linear(f(4, 8), f(6, 8), f(7, 8))
    with pytest.raises(ValueError, match="8 features"):
        lt.gated_linear(f(4, 9), f(6, 8), f(6, 8))
    with pytest.raises(ValueError, match="rows of 128"):
        lt.Int8Weight(6, 8, f(6, 8, dtype=torch.int8), f(6, dtype=torch.float32))
    with pytest.raises(ValueError, match="int8"):
        lt.Int8Weight(6, 8, f(6, 128, dtype=torch.uint8), f(6, dtype=torch.float32))
    with pytest.raises(ValueError, match="one for each row"):
        lt.Int8Weight(6, 8, f(6, 128, dtype=torch.int8), f(5, dtype=torch.float32))
    w = lt.Int8Weight(6, 8, f(6, 128, dtype=torch.int8), f(6, dtype=torch.float32))
    v = lt.Int8Weight(7, 8, f(7, 128, dtype=torch.int8), f(7, dtype=torch.float32))
    with pytest.raises(ValueError, match="features"):
        lt.int8_linear(f(4, 9), w)
    with pytest.raises(TypeError, match="float32 or bfloat16"):
        lt.int8_linear(f(4, 8, dtype=torch.float16), w)
    with pytest.raises(ValueError, match="up must have shape"):
        lt.int8_gated_linear(f(4, 8), w, v)
    with pytest.raises(ValueError, match="activation"):
        lt.int8_gated_linear(f(4, 8), w, w, "tanh")
    with pytest.raises(ValueError, match="w must have shape"):
        w.update(f(6, 9))


def test_sums_that_are_cut_need_their_memory():
    """m x n fp32 sums of either weight for every slice; none where something is kept, or for few
    tokens of a sum up to 4096 or of rows that tiles cannot read."""
    L = lib()
    need = L.lt_gated_forward_workspace_bytes(40, 64, 4096, 4096, 4096, 4096)
    assert need > 256 and need % (2 * 40 * 64 * 4) == 0
    assert L.lt_gated_forward_workspace_bytes(1, 64, 4160, 4160, 4160, 4160) > 256
    assert L.lt_gated_forward_workspace_bytes(16, 64, 4096, 4096, 4096, 4096) == 256
    kw = dict(m=40, n=64, k=4096, xs=4096, gs=4096, us=4096, stride=64)
    assert forward(**kw, saved=0, ws_bytes=need - 1) == lt.LT_ERR_WORKSPACE
    assert forward(**kw, saved=0, ws=0) == lt.LT_ERR_WORKSPACE
    assert forward(**kw, saved=0, ws=WS + 16) == lt.LT_ERR_WORKSPACE
    assert forward(**kw, saved=0, ws=4 * BASE) == lt.LT_ERR_INVALID_ARG  # out's
    need = L.lt_int8_matmul_workspace_bytes(40, 64, 9000)
    assert need > 256 and need % (40 * 64 * 4) == 0
    assert L.lt_int8_matmul_workspace_bytes(16, 64, 8192) == 256
    assert L.lt_int8_matmul_workspace_bytes(16, 64, 9000) > 256
    codes = 40 * 9088 + 256
    assert L.lt_int8_gated_workspace_bytes(40, 64, 9000) > codes + 2 * 40 * 64 * 4
