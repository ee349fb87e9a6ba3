"""Layers take tokens of every layout: any first address, transposed, broadcast, apart, in more
dimensions; the bits are those of a copy."""
import pytest
import torch

import paper_2608_11919_amd as lt

pytestmark = pytest.mark.gpu
DEV = "cuda"


def draw(shape, seed, dtype=torch.float32):
    gen = torch.Generator(DEV).manual_seed(seed)
    return torch.randn(shape, device=DEV, generator=gen).to(dtype)


LAYOUTS = {
    "rows from the second": lambda t, f, dt: draw((t + 1, f), 1, dt)[1:],
    "columns from the second": lambda t, f, dt: draw((t, f + 3), 2, dt)[:, 1:f + 1],
    "an odd address": lambda t, f, dt: draw((t * f + 1,), 3, dt)[1:].view(t, f),
    "transposed": lambda t, f, dt: draw((f, t), 4, dt).t(),
    "every other column": lambda t, f, dt: draw((t, 2 * f), 5, dt)[:, ::2],
    "one row for all": lambda t, f, dt: draw((1, f), 6, dt).expand(t, f),
    "one value for all": lambda t, f, dt: draw((1, 1), 7, dt).expand(t, f),
    "heads": lambda t, f, dt: draw((f // 3, t, 3), 8, dt).transpose(0, 1).reshape(t, -1)
    if f % 3 == 0 else draw((t, f), 8, dt),
    "overlapping rows": lambda t, f, dt: draw((t + f,), 9, dt).as_strided((t, f), (1, 1)),
}


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tokens", [1, 5, 16, 17, 40, 130])
@pytest.mark.parametrize("layout", LAYOUTS)
def test_tokens(layout, tokens, dtype):
    cols, rows = 333, 65
    x, dy = [LAYOUTS[layout](tokens, f, dtype) for f in (cols, rows)]
    weight = lt.Fp8Weight.from_master(draw((rows, cols), 20))
    # a copy at an address of its own
    xc, dyc = [t.clone(memory_format=torch.contiguous_format) for t in (x, dy)]
    assert xc.data_ptr() % 16 == 0 and xc.stride() == (cols, 1)
    assert torch.equal(lt.fp8_linear(x, weight), lt.fp8_linear(xc, weight))
    y, saved = lt.fp8_linear_forward(x, weight)
    y2, saved2 = lt.fp8_linear_forward(xc, weight)
    assert torch.equal(y, y2) and all(torch.equal(a, b) for a, b in zip(saved, saved2))
    got, want = [lt.fp8_linear_backward(d, saved, weight) for d in (dy, dyc)]
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_gradient_of_a_concatenation(dtype):
    """autograd hands each layer a view of the joined gradient, the second at an odd address."""
    w = draw((33, 70), 1, dtype).requires_grad_()
    weight = lt.Fp8Weight.from_master(w.detach())
    a, b = [draw((5 + i, 70), 2 + i, dtype).requires_grad_() for i in range(2)]
    c = draw((11, 33), 5, dtype)
    lin = lambda t: lt.Fp8Linear.apply(t, w, weight)
    got = torch.autograd.grad((torch.cat([lin(a), lin(b)], 0) * c).sum(), (a, b, w))
    want_a = torch.autograd.grad((lin(a) * c[:5]).sum(), (a, w))
    want_b = torch.autograd.grad((lin(b) * c[5:].clone()).sum(), (b, w))
    assert torch.equal(got[0], want_a[0]) and torch.equal(got[1], want_b[0])
    assert torch.equal(got[2], want_a[1] + want_b[1])


def test_transposed_tokens_through_autograd():
    w = draw((65, 96), 1).requires_grad_()
    weight = lt.Fp8Weight.from_master(w.detach())
    x = draw((96, 40), 2).requires_grad_()
    got = torch.autograd.grad(lt.Fp8Linear.apply(x.t(), w, weight).square().sum(), (x, w))
    xt = x.detach().t().contiguous().requires_grad_()
    want = torch.autograd.grad(lt.Fp8Linear.apply(xt, w, weight).square().sum(), (xt, w))
    assert torch.equal(got[0], want[0].t()) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("layout", [k for k in LAYOUTS if k != "heads"])
def test_weights(layout):
    w = LAYOUTS[layout](130, 77, torch.float32)
    copy = w.clone(memory_format=torch.contiguous_format)
    weight, want = lt.Fp8Weight.from_master(w), lt.Fp8Weight.from_master(copy)
    other = lt.Fp8Weight.empty(130, 77, DEV)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    other.update(w, stream=stream)
    stream.synchronize()
    for name in ("codes", "scales", "codes_t", "scales_t"):
        assert torch.equal(getattr(weight, name), getattr(want, name))
        assert torch.equal(getattr(other, name), getattr(want, name))


@pytest.mark.parametrize("shape", [(2, 3, 0), (0, 3, 0), (0, 3, 7), (40, 1, 0), (0,), (7,), (1, 1, 1)])
@pytest.mark.parametrize("rows", [0, 5])
def test_dimensions_of_zero_and_more_than_two(shape, rows):
    cols = shape[-1]
    x, dy = draw(shape, 1), draw(shape[:-1] + (rows,), 2)
    weight = lt.Fp8Weight.from_master(draw((rows, cols), 3))
    tokens = 1
    for n in shape[:-1]:
        tokens *= n
    x2, dy2 = x.reshape(tokens, cols), dy.reshape(tokens, rows)
    y, saved = lt.fp8_linear_forward(x, weight, out_dtype=torch.float32)
    y2, saved2 = lt.fp8_linear_forward(x2, weight, out_dtype=torch.float32)
    assert y.shape == shape[:-1] + (rows,) and torch.equal(y.reshape(tokens, rows), y2)
    assert torch.equal(lt.fp8_linear(x, weight, out_dtype=torch.float32), y)
    dx, dw = lt.fp8_linear_backward(dy, saved, weight)
    dx2, dw2 = lt.fp8_linear_backward(dy2, saved2, weight)
    assert dx.shape == shape and torch.equal(dx.reshape(tokens, cols), dx2)
    assert torch.equal(dw, dw2) and dw.shape == (rows, cols)
    if cols == 0:
        assert not y.any()
    if tokens == 0:
        assert not dw.any()
