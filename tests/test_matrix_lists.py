"""Rows and columns of matrix lists, read natively or one by one, and the checks of the matrix
operators that need no device."""
import ctypes

import pytest
import torch

import paper_2608_11919_amd as lt
from paper_2608_11919_amd import lazytrain as binding
from paper_2608_11919_amd import muon

lt.lib()


def _words(b):
    return list((ctypes.c_int64 * (len(b) // 8)).from_buffer_copy(b))


class Sub(torch.Tensor):
    pass


@pytest.mark.parametrize("matrices", [
    [], (), [torch.zeros(3, 4)], [torch.zeros(0, 7), torch.zeros(5, 1)],
    (torch.nn.Parameter(torch.zeros(2, 9)), torch.zeros(1, 1)), [torch.zeros(6, 8).t()]], ids=str)
def test_sides_of_plain_matrices(matrices):
    rows, cols = binding._lists.sides(matrices)
    assert _words(rows) == [m.shape[0] for m in matrices]
    assert _words(cols) == [m.shape[1] for m in matrices]
    assert muon._sides(matrices, "m") == (rows, cols)


@pytest.mark.parametrize("matrices", [[torch.zeros(3)], [torch.zeros(2, 2), torch.zeros(1, 2, 3)],
                                      [torch.zeros(2, 2), 5], [torch.zeros(2, 2).as_subclass(Sub)],
                                      "ab", None], ids=str)
def test_anything_else_is_left_to_the_checks(matrices):
    assert binding._lists.sides(matrices) is None


def test_a_tensor_subclass_is_read_one_by_one():
    rows, cols = muon._sides([torch.zeros(2, 3).as_subclass(Sub)], "m")
    assert _words(rows) == [2] and _words(cols) == [3]
    with pytest.raises(ValueError):
        muon._sides([torch.zeros(3)], "m")


def test_workspace_sizes():
    assert lt.lt_orthogonalize_workspace_bytes([], []) > 0
    assert lt.lt_orthogonalize_workspace_bytes([0, 5], [3, 0]) > 0
    assert lt.lt_orthogonalize_workspace_bytes([-1], [3]) == 0
    assert lt.lt_orthogonalize_workspace_bytes([1 << 23], [3]) == 0
    assert lt.lt_muon_workspace_bytes([64], [64], 100) == 0
    one = lt.lt_muon_workspace_bytes([4096], [4096], 4096)
    # X in three layouts twice and three n x n matrices in fp16, the update in fp32
    assert one >= 4096 * 4096 * (6 * 2 + 3 * 2 + 4)
    # a long list is worked on in batches that share the memory
    many = lt.lt_muon_workspace_bytes([4096] * 40, [4096] * 40, 4096)
    assert many < 9 * one
    L = lt.lib()
    assert L.lt_orthogonalize_workspace_bytes(None, None, 2) == 0
    assert L.lt_fp8_matmul_workspace_bytes(4, 4, 4) > 0
    assert L.lt_fp8_linear_workspace_bytes(100, 4, 300) >= 100 * 384 + 100 * 4
    assert (L.lt_fp8_code_pitch(1), L.lt_fp8_code_pitch(128), L.lt_fp8_code_pitch(129)) == \
        (128, 128, 256)
    assert (L.lt_fp8_scale_pitch(1), L.lt_fp8_scale_pitch(512), L.lt_fp8_scale_pitch(513)) == \
        (4, 4, 8)
    assert [lt.lt_fp8_code_pitch(c) for c in (0, 1, 300)] == [0, 128, 384]
    assert [lt.lt_fp8_scale_pitch(c) for c in (0, 1, 513)] == [0, 4, 8]


def test_argument_errors_without_a_device():
    """Checks run before any pointer or device use."""
    L = lt.lib()
    one = lambda i: (ctypes.c_void_p * 1)(0x1000000 * (i + 1))
    side = (ctypes.c_int64 * 1)(64)

    def orth(src=one(0), in_dtype=0, out=one(1), out_dtype=0, rows=side, cols=side, n=1, steps=5):
        return L.lt_orthogonalize(src, in_dtype, out, out_dtype, rows, cols, n, steps, None, 0, None)

    assert orth() == lt.LT_ERR_WORKSPACE  # the arguments are fine, no workspace is given
    assert orth(n=0) == lt.LT_ERR_WORKSPACE
    assert orth(n=-1) == lt.LT_ERR_INVALID_ARG
    assert orth(rows=None) == lt.LT_ERR_INVALID_ARG
    assert orth(rows=(ctypes.c_int64 * 1)(1 << 23)) == lt.LT_ERR_INVALID_ARG
    assert orth(in_dtype=2) == lt.LT_ERR_INVALID_ARG
    assert orth(out_dtype=-1) == lt.LT_ERR_INVALID_ARG
    assert orth(steps=0) == orth(steps=65) == lt.LT_ERR_INVALID_ARG
    assert orth(src=(ctypes.c_void_p * 1)(None)) == lt.LT_ERR_INVALID_ARG
    assert orth(src=(ctypes.c_void_p * 1)(0x1000008)) == lt.LT_ERR_ALIGNMENT
    assert orth(out=one(0)) == lt.LT_ERR_INVALID_ARG and b"overlap" in L.lt_last_error()

    def step(block=256, code_map=0, lr=1e-3, momentum=0.9, wd=0.0, rms=0.2, steps=5, ma=one(3),
             wb=None, coef=None):
        return L.lt_muon_step(one(0), one(1), 0, one(2), ma, wb, side, side, 1, block, code_map, lr,
                              momentum, 1, wd, rms, steps, coef, None, None, None, 0, None)

    assert step() == lt.LT_ERR_WORKSPACE
    for bad in (dict(block=100), dict(code_map=2), dict(lr=-1.0), dict(lr=float("inf")),
                dict(momentum=1.0), dict(momentum=float("nan")), dict(wd=-0.1), dict(rms=0.0),
                dict(steps=0), dict(ma=(ctypes.c_void_p * 1)(None)), dict(ma=one(0))):
        assert step(**bad) == lt.LT_ERR_INVALID_ARG, bad
    assert step(wb=(ctypes.c_void_p * 1)(0x9000002)) == lt.LT_ERR_ALIGNMENT
    assert step(coef=ctypes.c_void_p(0x9000002)) == lt.LT_ERR_ALIGNMENT

    p = ctypes.c_void_p(0x1000000)
    quantize = lambda x=p, dtype=0, rows=4, cols=4, stride=4, c=p, s=p, ct=None, st=None: \
        L.lt_fp8_quantize(x, dtype, rows, cols, stride, 0, c, s, ct, st, None)
    assert quantize(rows=0) == lt.LT_OK
    for bad in (dict(dtype=3), dict(rows=-1), dict(stride=3), dict(s=None), dict(ct=p),
                dict(x=None), dict(c=None, s=None), dict(rows=1 << 31)):
        assert quantize(**bad) == lt.LT_ERR_INVALID_ARG, bad
    assert quantize(x=ctypes.c_void_p(0x1000004)) == lt.LT_ERR_ALIGNMENT

    matmul = lambda m=100, n=100, k=1000, a=p, out=p, dtype=0, stride=100: L.lt_fp8_matmul(
        a, p, p, p, m, n, k, out, dtype, stride, None, 0, None)
    assert matmul() == lt.LT_ERR_WORKSPACE  # a cut sum needs one
    assert matmul(m=0) == lt.LT_OK
    for bad in (dict(m=-1), dict(k=1 << 23), dict(stride=99), dict(dtype=2), dict(a=None),
                dict(out=None)):
        assert matmul(**bad) == lt.LT_ERR_INVALID_ARG, bad
    assert matmul(out=ctypes.c_void_p(0x1000004)) == lt.LT_ERR_ALIGNMENT

    linear = lambda x=p, dtype=0, xs=1000, m=100, out_dtype=1, stride=100: L.lt_fp8_linear(
        x, dtype, xs, p, p, m, 100, 1000, p, out_dtype, stride, None, 0, None)
    assert linear() == lt.LT_ERR_WORKSPACE and linear(m=0) == lt.LT_OK
    for bad in (dict(x=None), dict(dtype=2), dict(xs=999), dict(out_dtype=5), dict(stride=10)):
        assert linear(**bad) == lt.LT_ERR_INVALID_ARG, bad
