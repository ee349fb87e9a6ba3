"""Fp8Linear in a graph of autograd's: first derivatives of the weight that the forward pass read,
or an error."""
import pytest
import torch

import paper_2608_11919_amd as lt

pytestmark = pytest.mark.gpu
DEV = "cuda"


def draw(shape, seed, dtype=torch.float32):
    gen = torch.Generator(DEV).manual_seed(seed)
    return torch.randn(shape, device=DEV, generator=gen).to(dtype)


def layer(tokens=5, cols=96, rows=72, dtype=torch.float32):
    """x, w and the 8-bit weight."""
    x = draw((tokens, cols), 1, dtype).requires_grad_()
    w = draw((rows, cols), 2, dtype).requires_grad_()
    return x, w, lt.Fp8Weight.from_master(w.detach())


# ------------------------------------------------------------ second derivatives

@pytest.mark.parametrize("loss", [lambda y, t: y.square().sum(), lambda y, t: y.sum(),
                                  lambda y, t: (t * y).sum()], ids=["square", "sum", "factor"])
def test_second_derivatives_are_refused(loss):
    """A penalty on a gradient, with another path beside the layer: never a number."""
    x, w, weight = layer()
    t = draw((1,), 3).requires_grad_()
    for wanted in (x, w):
        with pytest.raises(RuntimeError, match="first derivatives"):
            y = lt.Fp8Linear.apply(x, w, weight)
            g, = torch.autograd.grad(loss(y, t) + x.pow(3).sum() + w.pow(3).sum(), wanted,
                                     create_graph=True)
            g.square().sum().backward()


def test_gradients_that_are_constant_may_be_part_of_a_graph():
    """x alone needs a gradient of a linear function: dx depends on nothing that does."""
    x, w, weight = layer()
    want, = torch.autograd.grad(lt.Fp8Linear.apply(x, w, weight).sum(), x)
    y = lt.Fp8Linear.apply(x, w.detach(), weight)
    g, = torch.autograd.grad(y.sum() + x.pow(3).sum(), x, create_graph=True)
    assert torch.equal(g.detach(), want + 3 * x.detach().square())
    second, = torch.autograd.grad(g.sum(), x)
    assert torch.allclose(second, 6 * x.detach())
