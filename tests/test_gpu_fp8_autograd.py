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


# ------------------------------------------------------- a weight that changed since

def updated(weight, w):
    weight.update(w.detach() * 2)


def requantized(weight, w):
    lt.lt_fp8_quantize(w.detach() * 2, codes_t=weight.codes_t, scales_t=weight.scales_t,
                       square=True)


def written(weight, w):
    weight.codes_t.zero_()


@pytest.mark.parametrize("change", [updated, requantized, written])
def test_a_weight_that_changed_since_the_forward_pass(change):
    x, w, weight = layer()
    y = lt.Fp8Linear.apply(x, w, weight)
    y.sum().backward(retain_graph=True)
    change(weight, w)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_a_weight_updated_between_steps():
    """Forward, backward, update, and again: as with weights of their own."""
    x, w, weight = layer(33, 200, 130, torch.bfloat16)
    for turn in range(3):
        master = draw(w.shape, 50 + turn)
        weight.update(master)
        got = torch.autograd.grad(lt.Fp8Linear.apply(x, w, weight).square().sum(), (x, w))
        fresh = lt.Fp8Weight.from_master(master)
        want = torch.autograd.grad(lt.Fp8Linear.apply(x, w, fresh).square().sum(), (x, w))
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_weights_are_updated_in_inference_mode_too():
    x, w, weight = layer()
    with torch.inference_mode():
        weight.update(w)
        other = lt.Fp8Weight.from_master(w)
        other.update(w)
        assert torch.equal(lt.fp8_linear(x, weight), lt.fp8_linear(x, other))
    lt.Fp8Linear.apply(x, w, weight).sum().backward()


# ------------------------------------------------------------------ refusals

def test_a_weight_without_transposed_codes_is_refused_at_once():
    x, w, weight = layer()
    bare = lt.Fp8Weight.from_master(w.detach(), transposed=False)
    with pytest.raises(ValueError, match="transposed"):
        lt.Fp8Linear.apply(x, w, bare)
    # the gradient for w does not read them
    got, = torch.autograd.grad(lt.Fp8Linear.apply(x.detach(), w, bare).square().sum(), w)
    want, = torch.autograd.grad(lt.Fp8Linear.apply(x.detach(), w, weight).square().sum(), w)
    assert torch.equal(got, want)


def test_a_weight_whose_gradient_has_no_type_is_refused_at_once():
    x, w, weight = layer()
    with pytest.raises(TypeError):
        lt.Fp8Linear.apply(x, w.detach().half().requires_grad_(), weight)
    with pytest.raises(ValueError):
        lt.Fp8Linear.apply(x, w.detach()[:8], weight)


# ---------------------------------------------------------- only what is asked for

@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("asked", [(True, False), (False, True), (False, False), (True, True)])
def test_only_the_layouts_and_products_that_are_asked_for(asked, dtype, monkeypatch):
    from paper_2608_11919_amd import fp8
    x, w, weight = layer(40, 300, 130, dtype)
    want = torch.autograd.grad(lt.Fp8Linear.apply(x, w, weight).square().sum(), (x, w))
    layouts, products = [], []
    quantize, matmul = fp8.lt_fp8_quantize, fp8.lt_fp8_matmul

    def count_layouts(t, codes=None, scales=None, codes_t=None, scales_t=None, **kw):
        layouts.append((codes is not None, codes_t is not None))
        quantize(t, codes, scales, codes_t, scales_t, **kw)

    def count_products(*args, **kw):
        products.append(args[5].shape)
        matmul(*args, **kw)

    monkeypatch.setattr(fp8, "lt_fp8_quantize", count_layouts)
    monkeypatch.setattr(fp8, "lt_fp8_matmul", count_products)
    x2, w2 = x.detach().requires_grad_(asked[0]), w.detach().requires_grad_(asked[1])
    y = lt.Fp8Linear.apply(x2, w2, weight)
    assert layouts == [(True, asked[1])] and products == [(40, 130)]
    if any(asked):
        y.square().sum().backward()
        assert layouts[1:] == [asked]
        assert products[1:] == [s for s, a in (((40, 300), asked[0]), ((130, 300), asked[1])) if a]
    for t, g, a in ((x2, want[0], asked[0]), (w2, want[1], asked[1])):
        assert (t.grad is None) if not a else torch.equal(t.grad, g)


def test_a_gradient_that_does_not_read_the_weight_survives_its_update():
    x, w, weight = layer()
    want, = torch.autograd.grad(lt.Fp8Linear.apply(x.detach(), w, weight).sum(), w)
    y = lt.Fp8Linear.apply(x.detach(), w, weight)
    updated(weight, w)
    got, = torch.autograd.grad(y.sum(), w)
    assert torch.equal(got, want)
