"""The matrix operators' refusals that need no GPU: arrays that overlap, strides and sizes that no
launch could take, lists that do not fit host memory.  Addresses are made up; every call here
returns before it looks at one."""
import ctypes
import os
import subprocess
import sys
import textwrap

import pytest

import paper_2608_11919_amd as lt
from paper_2608_11919_amd.lazytrain import lib

BASE = 1 << 40  # an address on every boundary, which nothing reads
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def quantize(x=BASE, rows=300, cols=200, stride=200, codes=2 * BASE, scales=3 * BASE, codes_t=0,
             scales_t=0):
    return lib().lt_fp8_quantize(x, lt.LT_DTYPE_BF16, rows, cols, stride, 0, codes, scales,
                                 codes_t, scales_t, None)


def matmul(a=BASE, a_scales=2 * BASE, b=3 * BASE, b_scales=4 * BASE, m=40, n=48, k=130,
           out=5 * BASE, stride=48):
    return lib().lt_fp8_matmul(a, a_scales, b, b_scales, m, n, k, out, lt.LT_DTYPE_F32, stride,
                               None, 0, None)


def linear(x=BASE, x_stride=130, w=2 * BASE, w_scales=3 * BASE, m=4, n=48, k=130, out=4 * BASE,
           stride=48):
    return lib().lt_fp8_linear(x, lt.LT_DTYPE_F32, x_stride, w, w_scales, m, n, k, out,
                               lt.LT_DTYPE_F32, stride, None, 0, None)


@pytest.mark.parametrize("call", [
    # the last element of one array in the first 16 bytes of the other, either way round
    lambda: quantize(codes=BASE + (300 * 200 * 2 - 1) // 16 * 16),
    lambda: quantize(x=2 * BASE + (300 * 256 - 1) // 16 * 16),
    lambda: quantize(scales=2 * BASE + 300 * 256 - 4),
    lambda: quantize(codes_t=2 * BASE + 16, scales_t=4 * BASE),
    lambda: quantize(codes_t=5 * BASE, scales_t=3 * BASE + 4),
    lambda: matmul(out=BASE + 40 * 256 - 16),
    lambda: matmul(out=3 * BASE + 48 * 256 - 16),
    lambda: matmul(a=5 * BASE + (39 * 48 + 48) * 4 - 16),
    lambda: matmul(a_scales=5 * BASE),
    lambda: matmul(b_scales=5 * BASE + 64),
    lambda: linear(out=BASE + ((3 * 130 + 130) * 4 - 1) // 16 * 16),
    lambda: linear(out=2 * BASE),
    lambda: linear(w_scales=4 * BASE),
])
def test_overlaps(call):
    assert call() == lt.LT_ERR_INVALID_ARG
    assert b"overlap" in lib().lt_last_error()


@pytest.mark.parametrize("call", [
    lambda: quantize(stride=199),
    lambda: quantize(stride=1 << 62),
    lambda: quantize(rows=(1 << 31) - 1, cols=129, stride=129),  # 2^25 blocks
    lambda: quantize(rows=1 << 31, cols=1, stride=1),
    lambda: matmul(stride=47),
    lambda: matmul(stride=1 << 60),
    lambda: matmul(m=1 << 28, stride=48),
    lambda: matmul(m=1 << 22, n=1 << 22, stride=1 << 22),        # 2^28 tiles
    lambda: matmul(k=1 << 23),
    lambda: linear(x_stride=129),
    lambda: linear(x_stride=1 << 61),
    lambda: linear(n=1 << 28, stride=1 << 28),
])
def test_sizes(call):
    assert call() == lt.LT_ERR_INVALID_ARG


def test_lists_that_do_not_fit_host_memory():
    """With little address space left, the copies a call makes of its lists cannot be allocated:
    an error comes back, and the process lives."""
    code = textwrap.dedent("""
        import ctypes, resource
        import numpy as np
        import paper_2608_11919_amd as lt
        from paper_2608_11919_amd.lazytrain import lib
        L = lib()
        K = 1 << 26
        rows = np.zeros(K, dtype=np.int64)
        ptrs = np.zeros(K, dtype=np.int64)
        as_p = lambda a, t: ctypes.cast(a.ctypes.data, t)
        used = int(open("/proc/self/statm").read().split()[0]) * resource.getpagesize()
        resource.setrlimit(resource.RLIMIT_AS, (used + (64 << 20),) * 2)
        size = L.lt_orthogonalize_workspace_bytes
        args = size.argtypes
        got = size(as_p(rows, args[0]), as_p(rows, args[1]), K)
        assert got == 0, got
        size = L.lt_muon_workspace_bytes
        assert size(as_p(rows, size.argtypes[0]), as_p(rows, size.argtypes[1]), K, 256) == 0
        call = L.lt_orthogonalize
        t = call.argtypes
        rc = call(as_p(ptrs, t[0]), 0, as_p(ptrs, t[2]), 0, as_p(rows, t[4]), as_p(rows, t[5]), K,
                  5, None, 0, None)
        assert rc == lt.LT_ERR_HOST, rc
        assert b"memory" in L.lt_last_error()
        print("alive")
    """)
    env = dict(os.environ, PYTHONPATH=ROOT)
    got = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=100,
                         env=env)
    assert got.returncode == 0 and "alive" in got.stdout, got.stderr[-2000:]
