"""Captured orthogonalisations and Muon steps with the binding's own workspace: every replay gives
what an eager call gives, whatever calls of other lists came in between, and writes no memory
but its own."""
import pytest
import torch

import paper_2608_11919_amd as lt
from paper_2608_11919_amd import lazytrain as binding

pytestmark = pytest.mark.gpu
DEV = "cuda"
SHAPES = [(200, 333), (128, 700), (300, 260), (16, 900), (60, 70)]  # every way of working, both streams
MANY = [(8 + i, 40 + 3 * i) for i in range(30)]                     # descriptors of several launches


def draw(shapes, seed, scale=1e-2):
    gen = torch.Generator(DEV).manual_seed(seed)
    return [torch.randn(s, device=DEV, generator=gen) * scale for s in shapes]


def elsewhere(turn, stream):
    """A larger call of the same kinds on the stream, and tensors in whatever it freed."""
    big = draw([(1200 + 300 * turn, 2000)], 90 + turn)
    state = [torch.zeros(big[0].numel(), dtype=torch.int8, device=DEV)], \
        [torch.zeros(-(-big[0].numel() // 256), device=DEV)]
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        lt.lt_orthogonalize(big, [torch.empty_like(big[0])])
        lt.lt_muon_step(big, [big[0].clone()], *state, 256, lr=1e-3)
    stream.synchronize()
    with torch.cuda.stream(stream):
        others = [torch.full((1 << 22,), 7, dtype=torch.uint8, device=DEV) for _ in range(8)]
    stream.synchronize()
    return others


@pytest.mark.parametrize("warm", [False, True])
@pytest.mark.parametrize("shapes", [SHAPES, MANY], ids=["ways", "many"])
def test_orthogonalize(shapes, warm):
    us, stream = draw(shapes, 1), torch.cuda.Stream()
    out, want = [[torch.empty_like(u) for u in us] for _ in range(2)]
    torch.cuda.synchronize()
    if warm:
        lt.lt_orthogonalize(us, out, stream=stream)
        torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        lt.lt_orthogonalize(us, out)
    for turn in range(4):
        for u, v in zip(us, draw(shapes, 10 + turn)):
            u.copy_(v)
        for o in out:
            o.fill_(3.0)
        others = elsewhere(turn, stream)
        with torch.cuda.stream(stream):
            lt.lt_orthogonalize(us, want)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), turn
        assert all((o == 7).all() for o in others)


@pytest.mark.parametrize("dynamic", [False, True])
def test_muon_step(dynamic):
    def state(seed):
        w = draw(SHAPES, seed, 0.02)
        return (w, [torch.zeros(x.numel(), dtype=torch.int8, device=DEV) for x in w],
                [torch.zeros(-(-x.numel() // 256), device=DEV) for x in w])
    kw = dict(lr=1e-2, momentum=0.9, code_map=lt.LT_MAP_DYNAMIC if dynamic else lt.LT_MAP_LINEAR)
    grads, stream = draw(SHAPES, 3), torch.cuda.Stream()
    w, q, a = state(5)
    w2, q2, a2 = state(5)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        lt.lt_muon_step(w, grads, q, a, 256, **kw)
    for turn in range(4):
        for g, v in zip(grads, draw(SHAPES, 20 + turn)):
            g.copy_(v)
        others = elsewhere(turn, stream)
        graph.replay()
        torch.cuda.synchronize()
        lt.lt_muon_step(w2, grads, q2, a2, 256, **kw)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(w + q + a, w2 + q2 + a2)), turn
        assert all((o == 7).all() for o in others)


def test_a_workspace_that_a_graph_writes_is_never_taken_for_in_place():
    """Eager calls with one list around replays that write another's descriptors there."""
    us, vs = draw([(150, 200)], 1), draw([(90, 260), (70, 80)], 2)
    out, other, want = torch.empty_like(us[0]), [torch.empty_like(v) for v in vs], \
        [torch.empty_like(v) for v in vs]
    lt.lt_orthogonalize(vs, want)
    size = max(lt.lt_orthogonalize_workspace_bytes([150], [200]),
               lt.lt_orthogonalize_workspace_bytes([90, 70], [260, 80]))
    ws = torch.empty(size, dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lt.lt_orthogonalize(us, [out], workspace=ws)
    for _ in range(3):
        for o in other:
            o.zero_()
        graph.replay()
        lt.lt_orthogonalize(vs, other, workspace=ws)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(other, want))


def test_the_cached_workspace_of_a_captured_norm_is_kept():
    grads, stream = draw([(5000,), (70,)], 4), torch.cuda.Stream()
    S, S2 = [torch.zeros(1, dtype=torch.float64, device=DEV) for _ in range(2)]
    status, status2 = [torch.zeros(1, dtype=torch.int32, device=DEV) for _ in range(2)]
    torch.cuda.synchronize()
    lt.lt_grad_sqnorm(grads, S, status, stream=stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        lt.lt_grad_sqnorm(grads, S, status)
    held = len(binding._captured)
    assert held >= 1
    many = draw([(3000,)] * 4000, 5)
    torch.cuda.synchronize()
    lt.lt_grad_sqnorm(many, S2, status2, stream=stream)  # replaces the stream's workspace
    with torch.cuda.stream(stream):
        others = [torch.full((1 << 16,), 7, dtype=torch.uint8, device=DEV) for _ in range(64)]
    torch.cuda.synchronize()
    for turn in range(3):
        for g, v in zip(grads, draw([(5000,), (70,)], 30 + turn)):
            g.copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        lt.lt_grad_sqnorm(grads, S2, status2)
        assert status.item() == lt.LT_STATUS_OK and S.item() == S2.item()
        assert all((o == 7).all() for o in others)
