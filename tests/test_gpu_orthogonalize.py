"""lt_orthogonalize on the GPU against the polynomial in 64 bits.

Tolerances, in the 2-norm of the result.  An operand rounded to fp16 is at most 2^-12 of itself
off.  In a step X' = a X + B X the rounded operands are X (in both products), A and B, whose
terms weigh at most 4.775 * 1.446, 2.0315 * 1.446^2 and 2.81 against a result near 1: at most
15 * 2^-12 = 3.7e-3 a step if every rounding conspires, as in a matrix of one row, and the last
steps multiply it by |f'| < 1, so 1e-2 in all.  Over the sums of a matrix with 16 rows and
columns or more the roundings are independent and some four times smaller: 4e-3.  bf16 results
round by 2^-9 of an element more."""
import pytest
import torch

import paper_2608_11919_amd as lt

pytestmark = pytest.mark.gpu
DEV = "cuda"
A, B, C = 3.4445, -4.7750, 2.0315


def exact(u, steps=5):
    x = u.double()
    norm = torch.linalg.vector_norm(x)
    x = x / norm if norm > 0 else x
    for _ in range(steps):
        if x.shape[0] <= x.shape[1]:
            g = x @ x.t()
            x = A * x + (B * g + C * (g @ g)) @ x
        else:
            g = x.t() @ x
            x = A * x + x @ (B * g + C * (g @ g))
    return x


def matrix(rows, cols, seed, dtype=torch.float32, scale=1e-3):
    gen = torch.Generator(DEV).manual_seed(seed)
    x = torch.randn(rows, cols, device=DEV, generator=gen)
    if min(rows, cols) >= 8:  # a few strong directions over noise
        left = torch.randn(rows, 4, device=DEV, generator=gen)
        x = x + left @ torch.randn(4, cols, device=DEV, generator=gen)
    return (x * scale).to(dtype)


def bound(rows, cols, out_dtype):
    t = 4e-3 if min(rows, cols) >= 16 else 1e-2
    return t + (2.0 ** -9 if out_dtype == torch.bfloat16 else 0.0)


def check(u, got, steps=5):
    want = exact(u, steps)
    norm = torch.linalg.vector_norm(want).item()
    off = torch.linalg.vector_norm(got.double() - want).item()
    assert off <= bound(*u.shape, got.dtype) * norm, (tuple(u.shape), off / max(norm, 1e-300))


SHAPES = [(1, 1), (1, 5), (5, 1), (2, 2), (3, 1000), (1000, 3), (16, 300), (300, 16), (64, 64),
          (127, 129), (128, 128), (129, 65), (130, 130), (257, 513), (512, 300), (256, 1024),
          (1025, 384)]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtypes", [(torch.float32, torch.float32),
                                    (torch.bfloat16, torch.bfloat16)])
def test_one_matrix(shape, dtypes):
    u = matrix(*shape, 3, dtypes[0])
    out = torch.full(shape, 7.0, device=DEV, dtype=dtypes[1])
    lt.lt_orthogonalize([u], [out])
    check(u, out)


@pytest.mark.parametrize("dtypes", [(torch.float32, torch.bfloat16),
                                    (torch.bfloat16, torch.float32)])
def test_a_list_of_every_shape(dtypes):
    us = [matrix(*s, 10 + i, dtypes[0]) for i, s in enumerate(SHAPES + [(0, 4), (4, 0)] + SHAPES)]
    outs = [torch.empty(u.shape, device=DEV, dtype=dtypes[1]) for u in us]
    kept = [u.clone() for u in us]
    lt.lt_orthogonalize(us, outs)
    for u, o, k in zip(us, outs, kept):
        assert torch.equal(u, k)
        if u.numel():
            check(u, o)


@pytest.mark.parametrize("steps", [1, 2, 8])
def test_number_of_steps(steps):
    for shape in ((96, 200), (200, 96)):
        u = matrix(*shape, 5)
        out = torch.empty(shape, device=DEV)
        lt.lt_orthogonalize([u], [out], ns_steps=steps)
        # the bound is for results near 1; a single step leaves them small and is as exact
        check(u, out, steps)


def test_a_call_of_several_batches():
    shapes = [(4096, 16384), (64, 64), (9000, 8192), (200, 3000), (8192, 9000)]
    us = [matrix(*s, 20 + i, torch.bfloat16) for i, s in enumerate(shapes)]
    outs = [torch.empty(u.shape, device=DEV, dtype=torch.bfloat16) for u in us]
    lt.lt_orthogonalize(us, outs)
    for u, o in zip(us, outs):
        check(u, o)


def test_zero_nan_and_infinite_matrices_keep_to_themselves():
    us = [matrix(140, 90, 1), torch.zeros(33, 70, device=DEV), matrix(140, 90, 2),
          matrix(64, 200, 3), matrix(5, 5, 4)]
    us[2][17, 3] = float("nan")
    us[3][0, 199] = float("inf")
    outs = [torch.empty(u.shape, device=DEV) for u in us]
    lt.lt_orthogonalize(us, outs)
    check(us[0], outs[0])
    check(us[4], outs[4])
    assert torch.equal(outs[1], torch.zeros_like(outs[1]))
    assert torch.isnan(outs[2]).all() and torch.isnan(outs[3]).all()


@pytest.mark.parametrize("scale", [1e-30, 1e-20, 1e20, 1e30])
def test_scale_does_not_matter(scale):
    u = matrix(100, 150, 6, scale=1.0)
    a, b = torch.empty_like(u), torch.empty_like(u)
    lt.lt_orthogonalize([u], [a])
    lt.lt_orthogonalize([u * scale], [b])
    check(u * scale, b)
    assert torch.linalg.vector_norm(a - b) <= 4e-3 * torch.linalg.vector_norm(a)


def test_singular_values_end_near_one():
    u = matrix(300, 700, 8)
    out = torch.empty_like(u)
    lt.lt_orthogonalize([u], [out])
    s = torch.linalg.svdvals(out.double().cpu())
    assert 0.6 < s.min() and s.max() < 1.25


def test_same_bits_every_time_and_alone_or_in_a_list():
    us = [matrix(*s, 30 + i) for i, s in enumerate([(130, 257), (300, 40), (512, 512)])]
    outs = [[torch.empty_like(u) for u in us] for _ in range(2)]
    for o in outs:
        lt.lt_orthogonalize(us, o)
    for i, u in enumerate(us):
        alone = torch.empty_like(u)
        lt.lt_orthogonalize([u], [alone])
        assert torch.equal(outs[0][i], outs[1][i]) and torch.equal(outs[0][i], alone)


def test_on_another_stream_and_in_a_graph():
    u = matrix(200, 333, 9)
    want, got = torch.empty_like(u), torch.empty_like(u)
    lt.lt_orthogonalize([u], [want])
    ws = torch.empty(lt.lt_orthogonalize_workspace_bytes([200], [333]), dtype=torch.uint8,
                     device=DEV)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    lt.lt_orthogonalize([u], [got], workspace=ws, stream=s)
    s.synchronize()
    assert torch.equal(want, got)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        lt.lt_orthogonalize([u], [got], workspace=ws, stream=s)
    for seed in (40, 41, 42):
        u.copy_(matrix(200, 333, seed))
        got.zero_()
        graph.replay()
        torch.cuda.synchronize()
        lt.lt_orthogonalize([u], [want])
        torch.cuda.synchronize()
        assert torch.equal(want, got)


def test_refusals():
    u, out = matrix(8, 8, 1), torch.empty(8, 8, device=DEV)
    with pytest.raises(ValueError):
        lt.lt_orthogonalize([u], [])
    with pytest.raises(ValueError):
        lt.lt_orthogonalize([u.view(-1)], [out.view(-1)])
    with pytest.raises(ValueError):
        lt.lt_orthogonalize([u], [torch.empty(4, 16, device=DEV)])
    with pytest.raises(ValueError):
        lt.lt_orthogonalize([u.t()[:4]], [torch.empty(4, 8, device=DEV)])  # not contiguous
    with pytest.raises(TypeError):
        lt.lt_orthogonalize([u.half()], [out])
    with pytest.raises(ValueError):
        lt.lt_orthogonalize([u], [torch.empty(8, 8)])
    for steps in (0, -1, 65):
        with pytest.raises(lt.LazyTrainError):
            lt.lt_orthogonalize([u], [out], ns_steps=steps)
    with pytest.raises(lt.LazyTrainError):
        lt.lt_orthogonalize([u], [u])  # the result may not overlap the input
    with pytest.raises(ValueError):
        lt.lt_orthogonalize([u], [out], workspace=torch.empty(64, dtype=torch.uint8, device=DEV))
    lt.lt_orthogonalize([], [])
