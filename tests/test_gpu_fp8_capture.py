"""A captured linear layer replays what an eager call computes, also after a larger call has
replaced the cached workspace and other tensors have taken its memory."""
import pytest
import torch

import paper_2608_11919_amd as lt

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("tokens,cols,rows", [(1, 300, 520), (17, 1000, 300), (40, 9000, 200),
                                              (300, 700, 500)])
def test_replays(tokens, cols, rows):
    gen = torch.Generator(DEV).manual_seed(1)
    draw = lambda *s: torch.randn(*s, device=DEV, generator=gen)
    weight = lt.Fp8Weight.from_master(draw(rows, cols), transposed=False)
    x = draw(tokens, cols).bfloat16()
    lt.fp8_linear(x, weight)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        lt.fp8_linear(x, weight)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        y = lt.fp8_linear(x, weight)
    big = lt.Fp8Weight.from_master(draw(64, 20000), transposed=False)
    for turn in range(4):
        x.copy_(draw(tokens, cols))
        want = lt.fp8_linear(x, weight)
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):  # replaces the stream's cached workspace
            lt.fp8_linear(draw(512 * (turn + 1), 20000), big)
        stream.synchronize()
        others = [torch.full((1 << 20,), 7, dtype=torch.uint8, device=DEV) for _ in range(8)]
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want), turn
        assert all((o == 7).all() for o in others)
