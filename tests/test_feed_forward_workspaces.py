"""A workspace query of the feed-forward operators answers 256 only where nothing is looked at: what a
call does work in is larger, however small, so that a caller can tell the two apart.  Addresses are
made up; every call here returns before it looks at one."""
import pytest

import paper_2608_11919_amd as lt
from paper_2608_11919_amd.lazytrain import lib

BASE = 1 << 40  # an address on every boundary, which nothing reads


def matmul(m, n, k, ws, ws_bytes):
    return lib().lt_int8_matmul(BASE, 2 * BASE, 3 * BASE, 4 * BASE, m, n, k, 5 * BASE,
                                lt.LT_DTYPE_F32, n, ws, ws_bytes, None)


def forward(m, n, k, x_stride, saved, ws, ws_bytes):
    return lib().lt_gated_forward(BASE, x_stride, 2 * BASE, k, 3 * BASE, k, 0, m, n, k, 4 * BASE,
                                  lt.LT_DTYPE_BF16, n, saved, ws, ws_bytes, None)


@pytest.mark.parametrize("m,n,k", [(1, 1, 16384), (1, 2, 16384), (2, 1, 11008), (1, 2, 1 << 17),
                                   (1, 1, 8200), (17, 1, 5120)])
def test_few_integer_results_of_long_sums(m, n, k):
    need = lib().lt_int8_matmul_workspace_bytes(m, n, k)
    assert need > 256
    assert matmul(m, n, k, 0, 0) == lt.LT_ERR_WORKSPACE
    assert matmul(m, n, k, 6 * BASE, need - 1) == lt.LT_ERR_WORKSPACE


@pytest.mark.parametrize("m,n,k,x_stride,saved", [
    (1, 1, 8192, 8192, 0), (1, 2, 5120, 5120, 0), (1, 3, 5120, 5120, 0), (2, 1, 5120, 5120, 0),
    (1, 1, 4160, 4160, 0), (17, 1, 4160, 4160, 0),   # sums that are cut
    (17, 1, 8, 8, 0), (17, 1, 8, 8, 5 * BASE),       # packed operands: of all rows of x, or
    (18, 3, 64, 68, 0), (18, 3, 64, 68, 5 * BASE),   # of x alone
])
def test_few_gated_results(m, n, k, x_stride, saved):
    need = lib().lt_gated_forward_workspace_bytes(m, n, k, x_stride, k, k)
    assert need > 256
    assert forward(m, n, k, x_stride, saved, 0, 0) == lt.LT_ERR_WORKSPACE
    assert forward(m, n, k, x_stride, saved, 6 * BASE, 256) == lt.LT_ERR_WORKSPACE


@pytest.mark.parametrize("m,n,k", [(1, 1, 64), (1, 1, 8192), (16, 1, 8192), (300, 400, 128)])
def test_nothing_is_looked_at(m, n, k):
    assert lib().lt_int8_matmul_workspace_bytes(m, n, k) == 256
    if k <= 4096:
        assert lib().lt_gated_forward_workspace_bytes(m, n, k, k, k, k) == 256
