"""One or two results, for a few tokens, of sums long enough to be cut: what the slices' sums take
is less than a workspace's least unit.  Bounds as in test_gpu_gated.py; integers are bitwise."""
import pytest
import torch

import paper_2608_11919_amd as lt
from test_gpu_gated import Exact, inputs, near
from test_gpu_int8 import expected, matrix, product, quantize, same

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("m,n,k", [(1, 1, 16384), (1, 2, 16384), (2, 1, 11008), (1, 1, 8200),
                                   (1, 2, 20001), (17, 1, 5120)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_integers(m, n, k, dtype):
    a, b = matrix(m, k, 1, torch.float32), matrix(n, k, 2, torch.bfloat16)
    want = product(expected(a), expected(b), dtype)
    out = torch.empty(m, n, dtype=dtype, device=DEV)
    lt.lt_int8_matmul(*quantize(a), *quantize(b), k, out)
    assert same(out, want)
    assert same(lt.int8_linear(a, lt.Int8Weight.from_master(b), out_dtype=dtype), want)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device=DEV)
    lt.lt_int8_matmul(*quantize(a), *quantize(b), k, out.zero_(), workspace=ws)
    assert same(out, want)


@pytest.mark.parametrize("m,n,k", [(1, 1, 8192), (1, 2, 5120), (1, 3, 5120), (2, 1, 5120),
                                   (1, 1, 4160), (1, 1, 5001), (17, 1, 4160)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gated(m, n, k, dtype):
    x, gate, up, dh = inputs(m, n, k)
    e = Exact(x, gate, up, "silu")
    near(lt.gated_linear(x, gate, up, out_dtype=dtype), e.h, e.room, dtype)
    h, saved = lt.gated_linear_forward(x, gate, up, out_dtype=dtype)
    near(h, e.h, e.room, dtype)
    got = lt.gated_linear_backward(dh, saved, x, gate, up, dtype, dtype)
    for value, (want, room) in zip(got, e.gradients(dh).values()):
        near(value, want, room, dtype)


@pytest.mark.parametrize("m", [1, 2, 17])
def test_gated_with_one_packed_operand(m):
    """Rows of x that tiles cannot read as they are: their copies are 256 bytes for two tokens."""
    x, gate, up, dh = inputs(m, 40, 64)
    wide = torch.zeros(m, 68, dtype=torch.bfloat16, device=DEV)
    wide[:, :64] = x
    wide = wide[:, :64]
    h, saved = lt.gated_linear_forward(wide, gate, up)
    want = lt.gated_linear_forward(x, gate, up)
    assert torch.equal(h, want[0])
    assert torch.equal(lt.gated_linear(wide, gate, up), lt.gated_linear(x, gate, up))
    for a, b in zip(lt.gated_linear_backward(dh, saved, wide, gate, up),
                    lt.gated_linear_backward(dh, want[1], x, gate, up)):
        assert torch.equal(a, b)
