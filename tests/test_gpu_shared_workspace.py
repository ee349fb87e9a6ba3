"""One workspace for calls of every kind in stream order: a list call after one that overwrote its
descriptors writes them again."""
import pytest
import torch

import paper_2608_11919_amd as lt

pytestmark = pytest.mark.gpu
DEV = "cuda"


def draw(shape, seed):
    gen = torch.Generator(DEV).manual_seed(seed)
    return torch.randn(shape, device=DEV, generator=gen)


def layer(name):
    """Calls that write a workspace: x's codes, or partial sums (in slices)."""
    weight = lt.Fp8Weight.from_master(draw((200, 9000), 1), transposed=False)
    x = draw((40, 9000), 2)
    if name == "linear":
        return lambda ws: lt.fp8_linear(x, weight, workspace=ws)
    codes = torch.empty(40, lt.lt_fp8_code_pitch(9000), dtype=torch.uint8, device=DEV)
    scales = torch.empty(40, lt.lt_fp8_scale_pitch(9000), dtype=torch.uint8, device=DEV)
    lt.lt_fp8_quantize(x, codes, scales)
    out = torch.empty(40, 200, device=DEV)

    def product(ws):
        lt.lt_fp8_matmul(codes, scales, weight.codes, weight.scales, 9000, out, workspace=ws)
        return out.clone()
    return product


@pytest.mark.parametrize("name", ["linear", "matmul"])
@pytest.mark.parametrize("offset", [0, 256])
def test_orthogonalize_and_layers(name, offset):
    """With an offset the layer's workspace begins behind the other's tag."""
    call, us = layer(name), [draw((130, 300), 3), draw((20, 50), 4)]
    want, want_y = [torch.empty_like(u) for u in us], call(None)
    lt.lt_orthogonalize(us, want)
    ws = torch.empty(32 << 20, dtype=torch.uint8, device=DEV)
    part = ws[offset:]
    out = [torch.empty_like(u) for u in us]
    for _ in range(3):
        for o in out:
            o.zero_()
        lt.lt_orthogonalize(us, out, workspace=ws)
        assert torch.equal(call(part), want_y)
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_steps_and_layers():
    call = layer("linear")

    def state():
        w = [draw((130, 300), 5), draw((20, 50), 6)]
        return (w, [draw(x.shape, 7) for x in w],
                [torch.zeros(x.numel(), dtype=torch.int8, device=DEV) for x in w],
                [torch.zeros(-(-x.numel() // 256), device=DEV) for x in w])
    a, b = state(), state()
    ws = torch.empty(32 << 20, dtype=torch.uint8, device=DEV)
    for _ in range(3):
        lt.lt_muon_step(*a, 256, lr=1e-2)
        call(ws)
        lt.lt_muon_step(*b, 256, lr=1e-2, workspace=ws)
    for x, y in zip(a, b):
        assert all(torch.equal(s, t) for s, t in zip(x, y))


def test_a_captured_layer_writes_its_workspace_at_every_replay():
    call, us = layer("linear"), [draw((130, 300), 8)]
    want, out, want_y = torch.empty_like(us[0]), torch.empty_like(us[0]), call(None)
    lt.lt_orthogonalize(us, [want])
    ws = torch.empty(32 << 20, dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = call(ws)
    for _ in range(3):
        out.zero_()
        lt.lt_orthogonalize(us, [out], workspace=ws)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(y, want_y)
