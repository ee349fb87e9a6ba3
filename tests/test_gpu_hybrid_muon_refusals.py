"""A HybridMuon step that is refused changes nothing: neither AdamW's parameters nor Muon's, no
state and no count; the next step is the first one's twin."""
import pytest
import torch

import paper_2608_11919_amd as lt
from paper_2608_11919_amd import lazytrain as binding
from paper_2608_11919_amd import muon

pytestmark = pytest.mark.gpu
DEV = "cuda"
SHAPES = [(300, 128), (128,), (64, 48), (77,)]


def tensors(seed, scale):
    gen = torch.Generator(DEV).manual_seed(seed)
    return [torch.randn(s, device=DEV, generator=gen) * scale for s in SHAPES]


def make(slice_fraction):
    opt = lt.HybridMuon(tensors(1, 0.02), lr=1e-3, block_size=256, slice_fraction=slice_fraction,
                        bf16_copy=True)
    for c in opt.params_bf16:
        c.zero_()
    return opt


def snapshot(opt):
    return [t.clone() for t in opt.params + opt.params_bf16 + opt.m_codes + opt.v_codes +
            opt.m_absmax + opt.v_absmax + opt.exp_avg + opt.exp_avg_sq + opt.muon_codes +
            opt.muon_absmax]


def turned(opt, grads, monkeypatch):
    grads[0] = grads[0].t().contiguous()


def aliased(opt, grads, monkeypatch):
    grads[0] = opt.params[0]


def negative_rms(opt, grads, monkeypatch):
    opt.update_rms = -1.0


def no_steps(opt, grads, monkeypatch):
    opt.ns_steps = 0


def no_memory(opt, grads, monkeypatch):
    real = binding._workspace

    def full(device, nbytes, workspace, stream, kind, *rest):
        if kind == "muon":
            raise torch.cuda.OutOfMemoryError("no room")
        return real(device, nbytes, workspace, stream, kind, *rest)

    monkeypatch.setattr(binding, "_workspace", full)
    if hasattr(muon, "_workspace"):
        monkeypatch.setattr(muon, "_workspace", full)


@pytest.mark.parametrize("slice_fraction", [None, 0.2])
@pytest.mark.parametrize("fault", [turned, aliased, negative_rms, no_steps, no_memory])
def test_a_refused_step(fault, slice_fraction, monkeypatch):
    opt, twin = make(slice_fraction), make(slice_fraction)
    for o in (opt, twin):
        o.step(tensors(10, 1e-2))
    opt.last_status()
    before = snapshot(opt)
    bad = tensors(11, 1e-2)
    kept = (opt.update_rms, opt.ns_steps)
    with monkeypatch.context() as m:
        fault(opt, bad, m)
        with pytest.raises((ValueError, lt.LazyTrainError, torch.cuda.OutOfMemoryError)):
            opt.step(bad)
    opt.update_rms, opt.ns_steps = kept
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(before, snapshot(opt)))
    for o in (opt, twin):
        o.step(tensors(11, 1e-2))
        assert o.last_status() == lt.LT_STATUS_OK and o.step_count == 2
    assert all(torch.equal(a, b) for a, b in zip(snapshot(opt), snapshot(twin)))
