"""The matrix operators from two host threads at once, on one stream and on two: every result is
that of the same call alone."""
import threading

import pytest
import torch

import paper_2608_11919_amd as lt
from paper_2608_11919_amd import lazytrain as binding

pytestmark = pytest.mark.gpu
DEV = "cuda"
# long and square matrices: the library's second stream takes part
LISTS = [[(130, 400), (200, 220), (300, 300), (16, 300)], [(140, 290), (260, 250), (700, 130), (40, 90)]]


def draw(shape, seed):
    gen = torch.Generator(DEV).manual_seed(seed)
    return torch.randn(shape, device=DEV, generator=gen)


def both(work, streams):
    """work(i) in two threads, each on its stream."""
    errors, gate = [], threading.Barrier(2)
    torch.cuda.synchronize()

    def run(i):
        try:
            with torch.cuda.stream(streams[i]):
                gate.wait()
                work(i)
        except Exception as e:  # reported below
            errors.append(e)

    threads = [threading.Thread(target=run, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors, errors


def streams_of(one):
    a = torch.cuda.Stream()
    return [a, a if one else torch.cuda.Stream()]


def test_a_thread_has_its_own_workspaces():
    got, stream = [None, None], torch.cuda.Stream()

    def work(i):
        got[i] = [binding._workspace(torch.device(DEV, 0), 5000, None, None, "threads")
                  for _ in range(2)]

    both(work, [stream, stream])
    assert got[0][0] is got[0][1] and got[1][0] is got[1][1]
    assert got[0][0].data_ptr() != got[1][0].data_ptr()


@pytest.mark.parametrize("one_stream", [True, False])
@pytest.mark.parametrize("tokens", [3, 40, 200])
def test_linear(tokens, one_stream):
    """40 tokens through 9000 values: quantizer, product in slices and join, three launches."""
    weight = lt.Fp8Weight.from_master(draw((130, 9000), 1), transposed=False)
    xs = [[draw((tokens, 9000), 10 * i + j) for j in range(4)] for i in range(2)]
    want = [[lt.fp8_linear(x, weight) for x in ts] for ts in xs]
    got = [[], []]

    def work(i):
        for r in range(100):
            got[i].append(lt.fp8_linear(xs[i][r % 4], weight))

    both(work, streams_of(one_stream))
    for i in range(2):
        for r, y in enumerate(got[i]):
            assert torch.equal(y, want[i][r % 4]), (i, r)


@pytest.mark.parametrize("one_stream", [True, False])
def test_orthogonalize(one_stream):
    us = [[draw(s, 20 + 5 * i + j) for j, s in enumerate(LISTS[i])] for i in range(2)]
    want = [[torch.empty_like(u) for u in us[i]] for i in range(2)]
    got = [[[torch.empty_like(u) for u in us[i]] for _ in range(30)] for i in range(2)]
    for i in range(2):
        lt.lt_orthogonalize(us[i], want[i])

    def work(i):
        for out in got[i]:
            lt.lt_orthogonalize(us[i], out)

    both(work, streams_of(one_stream))
    for i in range(2):
        for r, out in enumerate(got[i]):
            assert all(torch.equal(a, b) for a, b in zip(out, want[i])), (i, r)


@pytest.mark.parametrize("one_stream", [True, False])
def test_muon_steps(one_stream):
    def state(i):
        w = [draw(s, 40 + 5 * i + j) * 0.02 for j, s in enumerate(LISTS[i])]
        return (w, [draw(s, 60 + 5 * i + j) for j, s in enumerate(LISTS[i])],
                [torch.zeros(x.numel(), dtype=torch.int8, device=DEV) for x in w],
                [torch.zeros(-(-x.numel() // 256), device=DEV) for x in w])
    alone, threaded = [state(i) for i in range(2)], [state(i) for i in range(2)]
    for i in range(2):
        for _ in range(20):
            lt.lt_muon_step(*alone[i], 256, lr=1e-2)

    def work(i):
        for _ in range(20):
            lt.lt_muon_step(*threaded[i], 256, lr=1e-2)

    both(work, streams_of(one_stream))
    for i in range(2):
        for a, b in zip(alone[i], threaded[i]):
            assert all(torch.equal(x, y) for x, y in zip(a, b)), i


def test_adamw_steps_on_one_stream():
    """The older list calls share the binding's workspaces."""
    def state(i):
        n = [5000 + 700 * i, 64, 20011]
        return ([draw((k,), 80 + i) for k in n], [draw((k,), 90 + i) for k in n],
                [torch.zeros(k, dtype=torch.int8, device=DEV) for k in n],
                [torch.zeros(-(-k // 256), device=DEV) for k in n],
                [torch.zeros(k, dtype=torch.uint8, device=DEV) for k in n],
                [torch.zeros(-(-k // 256), device=DEV) for k in n])
    alone, threaded = [state(i) for i in range(2)], [state(i) for i in range(2)]
    hyper = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01)
    for i in range(2):
        for t in range(1, 51):
            lt.lt_hybrid8bit_adamw_step(*alone[i], 256, step=t, **hyper)

    def work(i):
        for t in range(1, 51):
            lt.lt_hybrid8bit_adamw_step(*threaded[i], 256, step=t, **hyper)

    both(work, streams_of(True))
    for i in range(2):
        for a, b in zip(alone[i], threaded[i]):
            assert all(torch.equal(x, y) for x, y in zip(a, b)), i
