"""lt_muon_step on the GPU: momentum codes and scales bitwise against 32-bit arithmetic on the
host and the oracle's quantizer, weights against the step in 64 bits.

A weight is fma(-rate, O, w * decay): two roundings of 2^-24 of its terms, and rate times what
the orthogonalisation is off (4e-3 of O's 2-norm from 16 rows and columns, 1e-2 below, see
test_gpu_orthogonalize.py)."""
import math

import numpy as np
import pytest
import torch

import oracle
import paper_2608_11919_amd as lt
from test_gpu_orthogonalize import exact as orthogonal

pytestmark = pytest.mark.gpu
DEV = "cuda"
LR, WD, RMS = 1e-2, 0.1, 0.2


class Matrices:
    def __init__(self, shapes, block, dynamic, grad_dtype, seed=0):
        r = np.random.default_rng(seed)
        self.shapes, self.block, self.dynamic = shapes, block, dynamic
        self.w = [(r.standard_normal(s) * 0.02).astype(np.float32) for s in shapes]
        self.g = [torch.from_numpy((r.standard_normal(s) * 1e-3).astype(np.float32)).to(grad_dtype)
                  for s in shapes]
        self.codes = [r.integers(-128 if dynamic else -127, 128, math.prod(s)).astype(np.int8)
                      for s in shapes]
        self.absmax = [(r.random(-(-math.prod(s) // block)) * 4e-3 + 1e-4).astype(np.float32)
                       for s in shapes]

    def to_dev(self):
        dev = lambda xs: [torch.from_numpy(x.copy()).to(DEV) for x in xs]
        return dev(self.w), [g.to(DEV) for g in self.g], dev(self.codes), dev(self.absmax)

    def expected(self, coef, momentum, nesterov, steps=5):
        """[(weights in 64 bits, codes, absmax, allowed error of the weights)]"""
        f = np.float32
        out = []
        deq = oracle.dequantize_dynamic_signed if self.dynamic else oracle.dequantize_signed
        enc = oracle.quantize_dynamic_signed if self.dynamic else oracle.quantize_signed
        for w, g, q, a, (rows, cols) in zip(self.w, self.g, self.codes, self.absmax, self.shapes):
            n, b = w.size, self.block
            if n == 0:
                out.append((w.astype(np.float64), q, a, 0.0))
                continue
            m0 = np.concatenate([deq(q[i:i + b], a[i // b]) for i in range(0, n, b)])
            cg = (g.float().numpy().reshape(-1) * f(coef)) * f(1 - momentum)
            m1 = m0 * f(momentum) + cg
            u = m1 * f(momentum) + cg if nesterov else m1
            blocks = [enc(m1[i:i + b]) for i in range(0, n, b)]
            o = orthogonal(torch.from_numpy(u.reshape(rows, cols)).to(DEV), steps).cpu().numpy()
            rate = f(LR * RMS * math.sqrt(max(rows, cols)))
            want = w.astype(np.float64) * f(1 - LR * WD) - float(rate) * o
            off = float(rate) * (4e-3 if min(rows, cols) >= 16 else 1e-2) * np.linalg.norm(o) + \
                2.0 ** -23 * (np.linalg.norm(w) + float(rate) * np.linalg.norm(o))
            out.append((want, np.concatenate([x[0] for x in blocks]),
                        np.array([x[1] for x in blocks], np.float32), off))
        return out


def check(ms, dev, expect, copies=None):
    w, _, codes, absmax = dev
    for k, (want, q, a, off) in enumerate(expect):
        if want.size == 0:
            continue
        assert codes[k].cpu().numpy().tobytes() == q.tobytes(), k
        assert absmax[k].cpu().numpy().tobytes() == a.tobytes(), k
        assert np.linalg.norm(w[k].cpu().numpy() - want) <= off, k
        if copies is not None:
            assert torch.equal(copies[k].view(w[k].shape), w[k].to(torch.bfloat16))


SHAPES = [(1, 1), (3, 70), (64, 64), (129, 257), (300, 40), (16, 2048), (0, 7)]


@pytest.mark.parametrize("block", [64, 192, 512, 4096, 12288, 65536])
@pytest.mark.parametrize("dynamic", [False, True])
@pytest.mark.parametrize("grad", [torch.bfloat16, torch.float32])
def test_a_step(block, dynamic, grad):
    ms = Matrices(SHAPES, block, dynamic, grad, seed=block)
    dev = ms.to_dev()
    copies = [torch.zeros(s, dtype=torch.bfloat16, device=DEV) for s in SHAPES]
    coef = torch.full((1,), 0.37, device=DEV)
    kw = dict(lr=LR, weight_decay=WD, code_map=lt.LT_MAP_DYNAMIC if dynamic else lt.LT_MAP_LINEAR)
    lt.lt_muon_step(*dev, block, momentum=0.9, coef=coef, params_bf16=copies, **kw)
    check(ms, dev, ms.expected(0.37, 0.9, True), copies)
    # without Nesterov's look ahead, without clipping, no copies
    dev = ms.to_dev()
    lt.lt_muon_step(*dev, block, momentum=0.95, nesterov=False, **kw)
    check(ms, dev, ms.expected(1.0, 0.95, False))


@pytest.mark.parametrize("block", [256, 4096, 16384])
def test_momentum_without_memory(block):
    """momentum = 0: the plain orthogonalised gradient."""
    ms = Matrices([(200, 100), (64, 333)], block, False, torch.float32, seed=2)
    dev = ms.to_dev()
    lt.lt_muon_step(*dev, block, lr=LR, weight_decay=WD, momentum=0.0)
    check(ms, dev, ms.expected(1.0, 0.0, True))


def test_zero_gradient_and_zero_momentum_only_decay():
    ms = Matrices([(40, 60)], 256, False, torch.float32)
    w, g, q, a = ms.to_dev()
    g[0].zero_(), q[0].zero_(), a[0].zero_()
    before = w[0].clone()
    lt.lt_muon_step(w, g, q, a, 256, lr=LR, weight_decay=WD)
    assert torch.equal(w[0], before * torch.tensor(1 - LR * WD, dtype=torch.float32, device=DEV))
    assert not q[0].any() and not a[0].any()


@pytest.mark.parametrize("how", ["status", "stopped", "table"])
def test_a_skipped_step_writes_nothing_but_the_copy(how):
    ms = Matrices([(130, 70), (16, 500)], 512, True, torch.bfloat16)
    dev = ms.to_dev()
    kept = [[t.clone() for t in ts] for ts in dev]
    copies = [torch.zeros(s, dtype=torch.bfloat16, device=DEV) for s in ms.shapes]
    kw = {}
    if how == "status":
        kw["status"] = torch.ones(1, dtype=torch.int32, device=DEV)
    else:
        state = torch.empty(lt.lt_step_state_bytes(4), dtype=torch.uint8, device=DEV)
        lt.lt_step_state_init(state, 4, 0.9, 0.999, applied=4 if how == "table" else 0)
        if how == "stopped":
            state[24:25] = 1
        kw["step_state"] = state
    lt.lt_muon_step(*dev, 512, lr=LR, weight_decay=WD, code_map=lt.LT_MAP_DYNAMIC,
                    params_bf16=copies, **kw)
    for a, b in zip(dev, kept):
        for x, y in zip(a, b):
            assert torch.equal(x, y)
    for c, w in zip(copies, dev[0]):
        assert torch.equal(c, w.to(torch.bfloat16))


def test_a_step_state_that_applies():
    ms = Matrices([(130, 70)], 512, False, torch.bfloat16)
    dev = ms.to_dev()
    state = torch.empty(lt.lt_step_state_bytes(4), dtype=torch.uint8, device=DEV)
    lt.lt_step_state_init(state, 4, 0.9, 0.999, applied=3)
    lt.lt_muon_step(*dev, 512, lr=LR, weight_decay=WD, momentum=0.95, step_state=state,
                    status=torch.zeros(1, dtype=torch.int32, device=DEV))
    check(ms, dev, ms.expected(1.0, 0.95, True))


def test_refusals():
    ms = Matrices([(32, 64)], 256, False, torch.float32)
    w, g, q, a = ms.to_dev()
    ok = dict(lr=LR)
    for bad in (dict(lr=-1.0), dict(lr=float("nan")), dict(lr=LR, momentum=1.0),
                dict(lr=LR, momentum=-0.1), dict(lr=LR, weight_decay=-1.0),
                dict(lr=LR, update_rms=0.0), dict(lr=LR, ns_steps=0), dict(lr=LR, ns_steps=65),
                dict(lr=LR, code_map=2)):
        with pytest.raises(lt.LazyTrainError):
            lt.lt_muon_step(w, g, q, a, 256, **bad)
    for block in (0, 100, 65600):
        with pytest.raises((lt.LazyTrainError, ValueError)):
            lt.lt_muon_step(w, g, q, a, block, **ok)
    with pytest.raises(lt.LazyTrainError):  # weights may not alias the gradient
        lt.lt_muon_step(w, w, q, a, 256, **ok)
    with pytest.raises(ValueError):
        lt.lt_muon_step([w[0].view(-1)], g, q, a, 256, **ok)
    with pytest.raises(ValueError):
        lt.lt_muon_step(w, [g[0][:16]], q, a, 256, **ok)
    with pytest.raises(ValueError):
        lt.lt_muon_step(w, g, q, [a[0][:4]], 256, **ok)
    with pytest.raises(TypeError):
        lt.lt_muon_step([w[0].double()], g, q, a, 256, **ok)
    with pytest.raises(TypeError):
        lt.lt_muon_step(w, [g[0].half()], q, a, 256, **ok)
    lt.lt_muon_step([], [], [], [], 256, **ok)
