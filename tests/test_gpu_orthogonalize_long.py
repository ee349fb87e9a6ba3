"""Long matrices, whose Gram matrices are summed in slices, against the polynomial in 64 bits.

The tolerance is that of tests/test_gpu_orthogonalize.py for sides of 16 and more, 4e-3 of the
result's 2-norm (bf16 results 2^-9 more): slices only change the order of fp32 sums, whose error is
far below that of the fp16 operands."""
import pytest
import torch

import paper_2608_11919_amd as lt

pytestmark = pytest.mark.gpu
DEV = "cuda"
A, B, C = 3.4445, -4.7750, 2.0315


def exact(u, steps=5):
    x = u.double()
    x = x / torch.linalg.vector_norm(x)
    tall = x.shape[0] > x.shape[1]
    x = x.t() if tall else x
    for _ in range(steps):
        g = x @ x.t()
        x = A * x + (B * g + C * (g @ g)) @ x
    return x.t() if tall else x


def draw(rows, cols, seed):
    gen = torch.Generator(DEV).manual_seed(seed)
    x = torch.randn(rows, cols, device=DEV, generator=gen)
    left = torch.randn(rows, 4, device=DEV, generator=gen)
    return x + left @ torch.randn(4, cols, device=DEV, generator=gen)


def check(u, got, steps=5):
    want = exact(u, steps)
    off = (torch.linalg.vector_norm(got.double() - want) / torch.linalg.vector_norm(want)).item()
    assert off <= 4e-3 + (2.0 ** -9 if got.dtype == torch.bfloat16 else 0.0), (u.shape, off)


SHAPES = [(65, 1025), (1024, 66), (128, 2048), (100, 9000), (9001, 129), (200, 5003), (260, 4097),
          (640, 6000), (3000, 520), (128, 40000)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_one(shape, dtype):
    u = draw(*shape, 1).to(dtype)
    out = [torch.empty(shape, device=DEV, dtype=dtype) for _ in range(2)]
    lt.lt_orthogonalize([u], out[:1])
    lt.lt_orthogonalize([u], out[1:])
    check(u.float(), out[0])
    assert torch.equal(*out)


@pytest.mark.parametrize("steps", [1, 4, 5])
def test_lists_of_several_lengths(steps):
    """One number of slices for matrices of different lengths: short ones have fewer."""
    shapes = [(128, 17000), (130, 400), (70, 1200), (300, 300), (2100, 1000), (66, 66)]
    us = [draw(*s, i) for i, s in enumerate(shapes)]
    out = [torch.empty_like(u) for u in us]
    lt.lt_orthogonalize(us, out, ns_steps=steps)
    for u, o in zip(us, out):
        check(u, o, steps)


def test_nan_keeps_to_its_matrix():
    us = [draw(128, 5000, 1), draw(128, 5000, 2)]
    us[0][7, 4999] = float("nan")
    out = [torch.empty_like(u) for u in us]
    lt.lt_orthogonalize(us, out)
    assert out[0].isnan().all()
    check(us[1], out[1])
