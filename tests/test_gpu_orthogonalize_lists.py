"""Lists whose Gram matrices are summed in slices and whose steps are paired: the same list gives
the same bits on any stream, eager or captured; in another list a matrix's sums are cut
elsewhere, and its result may differ by the roundings, not more.

That difference is at most the sum of both results' distances from the polynomial, 4e-3 of the
2-norm each for noise with a few mild directions (tests/test_gpu_orthogonalize.py)."""
import pytest
import torch

import paper_2608_11919_amd as lt

pytestmark = pytest.mark.gpu
DEV = "cuda"
LISTS = [[(128, 5000), (128, 17000)], [(128, 5000)] * 40, [(300, 2000), (128, 5000), (512, 512)],
         [(1024, 9000), (640, 600), (70, 3000)]]


def draw(shapes, dtype):
    out = []
    for i, s in enumerate(shapes):
        gen = torch.Generator(DEV).manual_seed(10 + i)
        x = torch.randn(s, device=DEV, generator=gen)
        left = torch.randn(s[0], 4, device=DEV, generator=gen)
        out.append((x + left @ torch.randn(4, s[1], device=DEV, generator=gen)).to(dtype))
    return out


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shapes", LISTS, ids=["two lengths", "forty", "three ways", "mixed"])
def test_same_list_same_bits(shapes, dtype):
    us = draw(shapes, dtype)
    outs = [[torch.empty_like(u) for u in us] for _ in range(4)]
    lt.lt_orthogonalize(us, outs[0])
    lt.lt_orthogonalize(us, outs[1])
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    lt.lt_orthogonalize(us, outs[2], stream=stream)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lt.lt_orthogonalize(us, outs[3])
    graph.replay()
    torch.cuda.synchronize()
    for other in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(outs[0], other))


@pytest.mark.parametrize("shapes", LISTS, ids=["two lengths", "forty", "three ways", "mixed"])
def test_alone_and_in_a_list_within_the_roundings(shapes):
    us = draw(shapes, torch.float32)
    outs = [torch.empty_like(u) for u in us]
    lt.lt_orthogonalize(us, outs)
    for i in (0, len(us) - 1):
        alone = torch.empty_like(us[i])
        lt.lt_orthogonalize([us[i]], [alone])
        off = torch.linalg.vector_norm(alone.double() - outs[i].double())
        print(f"{shapes[i]}: {(off / torch.linalg.vector_norm(alone.double())).item():.1e}")
        assert off <= 8e-3 * torch.linalg.vector_norm(alone.double())
