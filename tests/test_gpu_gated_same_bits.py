"""h has the same bits whether a pass keeps results for the backward pass or not: a re-entrant
checkpoint's first pass, with gradients off, and its second, under gradients, then agree."""
import pytest
import torch
from torch.utils.checkpoint import checkpoint

import paper_2608_11919_amd as lt
from test_gpu_gated import Exact, inputs, near
from test_gpu_int8 import ROOM

pytestmark = pytest.mark.gpu
DEV = "cuda"

# few tokens, sums that are cut, both with rows that tiles cannot read, whole tiles of each size
SIZES = [(1, 1, 1), (1, 70, 2048), (16, 33, 1000), (5, 40, 128), (3, 257, 4096), (1, 70, 4160),
         (16, 33, 8192), (9, 33, 5001), (17, 130, 4096), (40, 67, 5001), (90, 1, 4100),
         (128, 1024, 5120), (200, 300, 2560), (500, 257, 4096), (1030, 8200, 70)]


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("act", list(ROOM))
def test_forward(m, n, k, act):
    x, gate, up, _ = inputs(m, n, k)
    for dtype in (torch.float32, torch.bfloat16):
        h, saved = lt.gated_linear_forward(x, gate, up, act, out_dtype=dtype)
        assert torch.equal(lt.gated_linear(x, gate, up, act, out_dtype=dtype), h)
    ts = [t.requires_grad_() for t in (x, gate, up)]
    kept = lt.GatedLinear.apply(*ts, act)
    with torch.no_grad():
        assert torch.equal(lt.GatedLinear.apply(*ts, act), kept)


@pytest.mark.parametrize("m,n,k", [s for s in SIZES if s[0] * s[1] < 100000])
@pytest.mark.parametrize("act", list(ROOM))
def test_what_is_kept(m, n, k, act):
    """The gradients from it; relu's with exact sums."""
    x, gate, up, dh = inputs(m, n, k, exact=act == "relu")
    want = Exact(x, gate, up, act).gradients(dh)
    h, saved = lt.gated_linear_forward(x, gate, up, act)
    got = lt.gated_linear_backward(dh, saved, x, gate, up, torch.float32, torch.float32)
    for value, (exact, room) in zip(got, want.values()):
        near(value, exact, room, torch.float32)


@pytest.mark.parametrize("m,n,k", [(9, 64, 2048), (40, 64, 5120)])
def test_checkpoint(m, n, k):
    x, gate, up, dh = inputs(m, n, k)
    ts = [t.requires_grad_() for t in (x, gate, up)]
    seen = []

    def block(*ts):
        seen.append(lt.GatedLinear.apply(*ts))
        return seen[-1] * 1

    y = checkpoint(block, *ts, use_reentrant=True)
    y.backward(dh)
    assert len(seen) == 2 and torch.equal(seen[0], seen[1])
    got = [t.grad for t in ts]
    for a, b in zip(got, torch.autograd.grad(lt.GatedLinear.apply(*ts), ts, dh)):
        assert torch.equal(a, b)


def test_bad_tokens_of_cut_sums_stay_alone():
    for m, k in ((9, 2048), (40, 5120)):
        x, gate, up, dh = inputs(m, 70, k)
        want, saved = lt.gated_linear_forward(x, gate, up)
        dx0 = lt.gated_linear_backward(dh, saved, x, gate, up)[0]
        x[m - 1, k - 1] = float("inf")
        h, saved = lt.gated_linear_forward(x, gate, up)
        dx, dg, du = lt.gated_linear_backward(dh, saved, x, gate, up)
        assert torch.equal(h[:m - 1], want[:m - 1]) and torch.equal(dx[:m - 1], dx0[:m - 1])
        assert not torch.isfinite(h[m - 1]).all() and torch.isnan(dx[m - 1]).any()


def test_captured():
    """A graph of a pass that keeps what a cut sum gives, replayed beside other work."""
    x, gate, up, dh = inputs(40, 64, 5120)
    stream = torch.cuda.Stream()

    def call():
        h, saved = lt.gated_linear_forward(x, gate, up, "gelu")
        return (h, *lt.gated_linear_backward(dh, saved, x, gate, up))

    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        call()
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        out = call()
    for turn in range(3):
        x.copy_(inputs(40, 64, 5120)[0] * (turn + 1) / 2)
        want = call()
        torch.cuda.synchronize()
        others = [torch.full((1 << 20,), 7, dtype=torch.uint8, device=DEV) for _ in range(8)]
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
        assert all((o == 7).all() for o in others)
