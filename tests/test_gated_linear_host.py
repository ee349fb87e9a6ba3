"""What GatedLinear decides before the library is called, on the CPU with the library's work left
out: which calls keep their results, and which are refused."""
import pytest
import torch
from torch.autograd import forward_ad

import paper_2608_11919_amd as lt
from paper_2608_11919_amd import gated


@pytest.fixture
def kept(monkeypatch):
    """Whether each call's results were kept."""
    calls = []

    def forward(x, gate, up, activation, out_dtype, keep, workspace):
        calls.append(keep)
        return x.new_zeros(*x.shape[:-1], gate.shape[0], dtype=out_dtype), \
            torch.zeros(0, dtype=torch.uint8)

    monkeypatch.setattr(gated, "_forward", forward)
    return calls


def tensors(requires_grad=False):
    return [torch.ones(s, dtype=torch.bfloat16).requires_grad_(requires_grad)
            for s in ((4, 8), (6, 8), (6, 8))]


@pytest.mark.parametrize("mode", [torch.no_grad, torch.enable_grad])
@pytest.mark.parametrize("which", range(3))
def test_a_tangent_is_refused(kept, mode, which):
    """No derivative is silently zero: there is none in forward mode."""
    with forward_ad.dual_level(), mode():
        ts = tensors()
        ts[which] = forward_ad.make_dual(ts[which], torch.ones_like(ts[which]))
        with pytest.raises(NotImplementedError):
            lt.GatedLinear.apply(*ts)


def test_plain_tensors_beside_duals_keep_nothing(kept):
    with forward_ad.dual_level(), torch.inference_mode():
        lt.GatedLinear.apply(*tensors(True))
    with forward_ad.dual_level(), torch.no_grad():
        y = lt.GatedLinear.apply(*tensors(True))
        assert not y.requires_grad and forward_ad.unpack_dual(y).tangent is None
    with torch.no_grad():
        lt.GatedLinear.apply(*tensors(True), "gelu")
    with torch.inference_mode():
        lt.GatedLinear.apply(*tensors(True), activation="gelu")
    assert kept == [False] * 4
    assert lt.GatedLinear.apply(*tensors(True)).requires_grad and kept[-1]
