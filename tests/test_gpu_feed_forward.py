"""The feed-forward block's operators as a program runs them: trained in bf16 through the gated
projections and a layer in 8-bit floating point, stepped by the optimizer, laid out in integers
and asked; captured into graphs, on other streams, with a workspace of the caller's."""
import pytest
import torch

import paper_2608_11919_amd as lt

pytestmark = pytest.mark.gpu
DEV = "cuda"


def draw(gen, *shape, scale=1.0):
    return torch.randn(*shape, device=DEV, generator=gen) * scale


def test_a_block_trained_and_asked():
    gen = torch.Generator(DEV).manual_seed(2)
    width, inner, tokens = 128, 320, 96
    masters = [draw(gen, inner, width, scale=width ** -0.5),
               draw(gen, inner, width, scale=width ** -0.5),
               draw(gen, width, inner, scale=inner ** -0.5)]
    opt = lt.HybridMuon(masters, lr=1e-2, weight_decay=0.0, max_norm=1.0, block_size=256,
                        bf16_copy=True, matrices=[True] * 3)
    for p, c in zip(opt.params, opt.params_bf16):
        c.copy_(p.view(-1))
    gate, up, down = (c.view(p.shape).requires_grad_()
                      for p, c in zip(opt.params, opt.params_bf16))
    weight = lt.Fp8Weight.from_master(masters[2])
    x, y = draw(gen, 2, tokens // 2, width).bfloat16(), draw(gen, 2, tokens // 2, width)
    for step in range(3):
        h = lt.GatedLinear.apply(x, gate, up)
        out = lt.Fp8Linear.apply(h, down, weight)
        loss = (out.float() - y).square().mean()
        grads = torch.autograd.grad(loss, (gate, up, down))
        assert all(torch.isfinite(g).all() and g.any() for g in grads)
        before = [p.clone() for p in opt.params]
        opt.step([g.contiguous() for g in grads])
        weight.update(opt.params[2])
        assert all(not torch.equal(a, b) for a, b in zip(before, opt.params))
        assert torch.equal(gate.detach(), opt.params[0].view(gate.shape).bfloat16())
    # the integers answer as near to the bf16 block as their steps allow: a code is off by half of
    # one in 127 of its row's largest, for Gaussian rows some 0.7% of a typical value, in each of
    # two operands of two layers
    ints = [lt.Int8Weight.from_master(p.view(s)) for p, s in
            zip(opt.params, (gate.shape, up.shape, down.shape))]
    for n in (1, 7, 40, tokens):
        t = x.view(tokens, width)[:n]
        wide = lt.gated_linear(t, gate.detach(), up.detach()).float() @ down.detach().float().t()
        short = lt.int8_linear(lt.int8_gated_linear(t, *ints[:2]), ints[2]).float()
        assert (short - wide).norm() <= 0.05 * wide.norm()
    ints[0].update(opt.params[0].view(gate.shape) * 2)
    assert not torch.equal(lt.int8_gated_linear(t, *ints[:2]).float(), short)


def calls(tokens, gen):
    """{name: (inputs that change, call)}"""
    n, k = 320, 200
    w = [draw(gen, n, k, scale=k ** -0.5) for _ in range(2)]
    ints = [lt.Int8Weight.from_master(v) for v in w]
    gate, up = (v.bfloat16() for v in w)
    x, dh = draw(gen, tokens, k).bfloat16(), draw(gen, tokens, n).bfloat16()

    def train():
        h, saved = lt.gated_linear_forward(x, gate, up, "gelu_tanh")
        return (h, *lt.gated_linear_backward(dh, saved, x, gate, up))

    return {"gated": ([x], lambda: (lt.gated_linear(x, gate, up),)),
            "train": ([x, dh], train),
            "int8": ([x], lambda: (lt.int8_linear(x, ints[0]),)),
            "int8_gated": ([x], lambda: (lt.int8_gated_linear(x, *ints),))}


@pytest.mark.parametrize("tokens", [1, 20, 300, 7000])
def test_captured_and_replayed(tokens):
    gen = torch.Generator(DEV).manual_seed(1)
    for name, (change, call) in calls(tokens, gen).items():
        stream = torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            call()
        stream.synchronize()
        graphs, outs = [], []
        for _ in range(2):  # two graphs of one call: neither writes where the other reads
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                outs.append(call())
            graphs.append(graph)
        for turn in range(3):
            for t in change:
                t.copy_(draw(gen, *t.shape))
            want = call()
            torch.cuda.synchronize()
            others = [torch.full((1 << 20,), 7, dtype=torch.uint8, device=DEV) for _ in range(8)]
            for graph in graphs:
                graph.replay()
            torch.cuda.synchronize()
            for got in outs:
                assert all(torch.equal(a, b) for a, b in zip(got, want)), (name, turn)
            assert all((o == 7).all() for o in others)


def test_a_captured_backward_pass_beside_an_eager_graph():
    """Refused while a graph of the same leaves, made on the default stream, lives; captured and
    replayed once that is gone."""
    gen = torch.Generator(DEV).manual_seed(3)
    x = draw(gen, 70, 64).bfloat16()
    gate, up = (draw(gen, 96, 64, scale=0.1).bfloat16().requires_grad_() for _ in range(2))
    dh = draw(gen, 70, 96).bfloat16()
    grads = lambda: torch.autograd.grad(lt.GatedLinear.apply(x, gate, up), (gate, up), dh)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        grads()
    stream.synchronize()
    eager = lt.GatedLinear.apply(x, gate, up)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        also = x + 1
        with pytest.raises(RuntimeError, match="holds the same leaf"):
            lt.GatedLinear.apply(x, gate, up)
    del graph, also
    wanted = torch.autograd.grad(eager, (gate, up), dh)
    del eager
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        got = grads()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, wanted))
    for turn in range(3):
        x.copy_(draw(gen, 70, 64))
        graph.replay()
        torch.cuda.synchronize()
        want = grads()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_other_streams_and_workspaces():
    gen = torch.Generator(DEV).manual_seed(4)
    for tokens in (20, 300):
        made = calls(tokens, gen)
        want = {name: call() for name, (_, call) in made.items()}
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in range(2)]
        got = []
        for turn in range(4):
            with torch.cuda.stream(streams[turn % 2]):
                got.append({name: call() for name, (_, call) in made.items()})
        torch.cuda.synchronize()
        for g in got:
            for name in want:
                assert all(torch.equal(a, b) for a, b in zip(g[name], want[name])), name
    # one workspace, call after call, also after a list call that keeps descriptors there
    x = draw(gen, 300, 200).bfloat16()
    ws = torch.empty(16 << 20, dtype=torch.uint8, device=DEV)
    w = [draw(gen, 320, 200, scale=0.1) for _ in range(2)]
    ints = [lt.Int8Weight.from_master(v) for v in w]
    gate, up = (v.bfloat16() for v in w)
    ones = [draw(gen, 100, 100)]
    out = [torch.empty(100, 100, device=DEV)]
    eager = torch.empty(100, 100, device=DEV)
    lt.lt_orthogonalize(ones, [eager])
    for _ in range(2):
        lt.lt_orthogonalize(ones, out, workspace=ws)
        assert torch.equal(out[0], eager)
        assert torch.equal(lt.gated_linear(x, gate, up, workspace=ws), lt.gated_linear(x, gate, up))
        lt.lt_orthogonalize(ones, out, workspace=ws)
        assert torch.equal(out[0], eager)
        assert torch.equal(lt.int8_linear(x, ints[0], workspace=ws), lt.int8_linear(x, ints[0]))
        assert torch.equal(lt.int8_gated_linear(x, *ints, workspace=ws),
                           lt.int8_gated_linear(x, *ints))


def test_results_do_not_change():
    gen = torch.Generator(DEV).manual_seed(5)
    for tokens in (20, 300, 7000):
        for name, (_, call) in calls(tokens, gen).items():
            want = call()
            for _ in range(3):
                assert all(torch.equal(a, b) for a, b in zip(call(), want)), name


def test_two_threads_at_once():
    """Each with a stream of its own, over shared weights."""
    import threading
    gen = torch.Generator(DEV).manual_seed(7)
    made = {tokens: calls(tokens, gen) for tokens in (3, 300)}
    want = {t: {name: call() for name, (_, call) in m.items()} for t, m in made.items()}
    torch.cuda.synchronize()
    wrong = []

    def work(tokens):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(20):
                for name, (_, call) in made[tokens].items():
                    got = call()
                    torch.cuda.current_stream().synchronize()
                    if not all(torch.equal(a, b) for a, b in zip(got, want[tokens][name])):
                        wrong.append((tokens, name))

    threads = [threading.Thread(target=work, args=(t,)) for t in (3, 300, 300)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(60)
    assert not any(t.is_alive() for t in threads) and not wrong, wrong
