"""The gated projections in bf16, forward and backward, against 64 bits.

Sums of bf16's products in fp32, in any order and with truncated additions, are off by at most
(k + 16) * 2^-23 of the sum of magnitudes; act moves by at most 1.13 times and act' by at most
0.8 times as much as g does (relu's derivative jumps: its cases have sums that are exact).  For what
fp32 adds in the activation see ROOM in test_gpu_int8.py.

dg and du are rounded to bf16 (half a step, 2^-8 of themselves), after a and b were kept in 24
bits (2^-17).  Over a sum these roundings are as good as independent: the bound is eight times the
deviation of the sum, 2^-8 / sqrt(3) of the root of the sum of squares, beside the sum's own
(s + 16) * 2^-23 of the sum of magnitudes over s products, and the result's rounding."""
import math

import pytest
import torch

import paper_2608_11919_amd as lt
from test_gpu_int8 import ROOM, activation

pytestmark = pytest.mark.gpu
DEV = "cuda"
HALF = 2.0 ** -8


def draw(rows, cols, seed, scale=1.0):
    gen = torch.Generator(DEV).manual_seed(seed)
    return (torch.randn(rows, cols, device=DEV, generator=gen) * scale).bfloat16()


def inputs(m, n, k, exact=False):
    """x, gate, up, dh; exact: small integers, whose sums fp32 holds."""
    if exact:
        gen = torch.Generator(DEV).manual_seed(9)
        whole = lambda r, c: torch.randint(-3, 4, (r, c), device=DEV, generator=gen).bfloat16()
        return whole(m, k), whole(n, k), whole(n, k), whole(m, n)
    w = 2 / math.sqrt(k)
    return draw(m, k, 1), draw(n, k, 2, w), draw(n, k, 3, w), draw(m, n, 4)


def slope(name, g):
    if name == "relu":
        return (g > 0).double()
    g = g.detach().requires_grad_()
    return torch.autograd.grad(activation(name, g).sum(), g)[0]


class Exact:
    """The formulas in 64 bits, and how far fp32 may be off."""

    def __init__(self, x, gate, up, act):
        x, gate, up = (t.double().cpu() for t in (x, gate, up))
        self.x, self.gate, self.up, self.act = x, gate, up, act
        k = x.shape[1]
        self.g, self.u = x @ gate.t(), x @ up.t()
        unit = (k + 16) * 2.0 ** -23
        self.dg = unit * (x.abs() @ gate.abs().t())
        self.du = unit * (x.abs() @ up.abs().t())
        self.b = activation(act, self.g)
        self.a = self.u * slope(act, self.g)
        self.h = self.b * self.u
        rest = ROOM[act](self.g) * 2.0 ** -24
        self.room = (1.13 * self.dg * (self.u.abs() + self.du) + self.b.abs() * self.du +
                     rest * self.h.abs())
        self.room_b = 1.13 * self.dg + (rest + 2.0 ** -17) * self.b.abs()
        jump = 0.0 if act == "relu" else 0.8
        # act' is a sum of terms of up to 1.13 and 0.5 |g|, each within the activation's room
        self.room_a = (jump * self.dg * self.u.abs() + 1.13 * self.du + 2.0 ** -17 * self.a.abs() +
                       rest * (1.13 + self.g.abs()) * self.u.abs())

    def gradients(self, dh):
        """{name: (value, bound before the result's rounding)}"""
        d = dh.double().cpu()
        dg, du = d * self.a, d * self.b
        off_g = d.abs() * self.room_a
        off_u = d.abs() * self.room_b
        m, n = d.shape

        def product(terms, count):
            value, flat, square, sizes = 0, 0, 0, 0
            for (v, off), w in terms:
                value = value + v @ w
                flat = flat + off @ w.abs() * (1 + HALF)
                square = square + (v * v) @ (w * w)
                sizes = sizes + v.abs() @ w.abs()
            return value, (flat + 8 * HALF / math.sqrt(3) * square.sqrt() +
                           (count + 16) * 2.0 ** -23 * sizes)

        return dict(dx=product([((dg, off_g), self.gate), ((du, off_u), self.up)], 2 * n),
                    dgate=product([((dg.t(), off_g.t()), self.x)], m),
                    dup=product([((du.t(), off_u.t()), self.x)], m))


def near(got, want, room, dtype):
    got = got.double().cpu()
    bound = room + torch.finfo(dtype).eps / 2 * (want.abs() + room) + 1e-36
    off = (got - want).abs()
    assert (off <= bound).all(), (off / bound).max()


SIZES = [(1, 1, 1), (1, 520, 300), (2, 17, 64), (16, 33, 1000), (17, 300, 127), (32, 64, 2048),
         (33, 65, 128), (64, 200, 3001), (65, 1, 65), (300, 257, 257), (129, 2100, 640),
         (1030, 8200, 70)]


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("act", list(ROOM))
def test_forward(m, n, k, act):
    x, gate, up, _ = inputs(m, n, k)
    e = Exact(x, gate, up, act)
    for dtype in (torch.float32, torch.bfloat16):
        near(lt.gated_linear(x, gate, up, act, out_dtype=dtype), e.h, e.room, dtype)
        h, saved = lt.gated_linear_forward(x, gate, up, act, out_dtype=dtype)
        near(h, e.h, e.room, dtype)
        assert saved.numel() == 6 * m * (-(-n // 8) * 8)


# Sums that are cut, and few tokens of long sums with rows of any place.
@pytest.mark.parametrize("m,n,k", [(1, 70, 4160), (16, 33, 8192), (9, 33, 5001), (17, 130, 4096),
                                   (40, 67, 5001), (90, 1, 4100), (200, 300, 2560),
                                   (500, 257, 4096)])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_long_sums(m, n, k, act):
    x, gate, up, _ = inputs(m, n, k)
    e = Exact(x, gate, up, act)
    for dtype in (torch.float32, torch.bfloat16):
        h = lt.gated_linear(x, gate, up, act, out_dtype=dtype)
        near(h, e.h, e.room, dtype)
        assert torch.equal(h, lt.gated_linear(x, gate, up, act, out_dtype=dtype))
    want = lt.gated_linear(x, gate, up, act)
    x[0, k - 1] = float("nan")
    got = lt.gated_linear(x, gate, up, act)
    assert torch.isnan(got[0]).all() and torch.equal(got[1:], want[1:])


@pytest.mark.parametrize("m", [5, 17])
def test_rows_far_apart(m):
    """Rows further apart than the tiles' offsets reach are copied."""
    far = torch.zeros(m, 1 << 22, dtype=torch.bfloat16, device=DEV)
    x, gate, up, dh = inputs(m, 40, 128)
    far[:, :128] = x
    assert torch.equal(lt.gated_linear(far[:, :128], gate, up), lt.gated_linear(x, gate, up))
    got, want = (lt.gated_linear_forward(t, gate, up) for t in (far[:, :128], x))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    for a, b in zip(lt.gated_linear_backward(dh, got[1], far[:, :128], gate, up),
                    lt.gated_linear_backward(dh, want[1], x, gate, up)):
        assert torch.equal(a, b)


BACKWARD = [(1, 1, 1), (1, 40, 70), (70, 33, 100), (64, 64, 64), (65, 130, 63), (301, 200, 515),
            (129, 1030, 128), (1100, 64, 64), (7000, 30, 40)]


@pytest.mark.parametrize("m,n,k", BACKWARD)
@pytest.mark.parametrize("act", list(ROOM))
def test_backward(m, n, k, act):
    x, gate, up, dh = inputs(m, n, k, exact=act == "relu")
    want = Exact(x, gate, up, act).gradients(dh)
    for dtype in (torch.bfloat16, torch.float32):
        d = dh.to(dtype)
        h, saved = lt.gated_linear_forward(x, gate, up, act)
        got = dict(zip(("dx", "dgate", "dup"),
                       lt.gated_linear_backward(d, saved, x, gate, up, dtype, dtype)))
        for name, (value, room) in want.items():
            near(got[name], value, room, dtype)


def test_large_backward():
    """Tiles of every size, and sums that are cut."""
    for m, n, k in [(2100, 2080, 2064), (600, 5000, 320), (6200, 200, 200)]:
        x, gate, up, dh = inputs(m, n, k)
        want = Exact(x, gate, up, "silu").gradients(dh)
        h, saved = lt.gated_linear_forward(x, gate, up)
        for name, got in zip(("dx", "dgate", "dup"),
                             lt.gated_linear_backward(dh, saved, x, gate, up)):
            near(got, *want[name], torch.bfloat16)


def test_largest_backward():
    """Both products with rounds of the largest tiles, each in its launch.  The roundings of dg and du
    and of the result are two, each with a deviation of at most 2^-8 / sqrt(3) of a value: over all
    elements a 2-norm of at most 2^-8 * sqrt(2 / 3) of the result's (what fp32 adds is far below the
    tenth that is left for it)."""
    m, n, k = 8190, 4100, 8200
    x, gate, up, dh = inputs(m, n, k)
    h, saved = lt.gated_linear_forward(x, gate, up)
    got = lt.gated_linear_backward(dh, saved, x, gate, up)
    xs, gs, us = x.double(), gate.double(), up.double()
    g, u = xs @ gs.t(), xs @ us.t()
    s = torch.sigmoid(g)
    near_h = (h.double() - g * s * u).norm() / (g * s * u).norm()
    assert near_h <= HALF / math.sqrt(3) * 1.1
    dg = dh.double() * u * (s + g * s * (1 - s))
    du = dh.double() * g * s
    for value, want in zip(got, (dg @ gs + du @ us, dg.t() @ xs, du.t() @ xs)):
        off = (value.double() - want).norm() / want.norm()
        assert off <= HALF * math.sqrt(2 / 3) * 1.1, off


@pytest.mark.parametrize("act", list(ROOM))
@pytest.mark.parametrize("which", range(3))
def test_differences(act, which):
    """The gradient along a direction against central differences of the forward pass in fp32.  With
    steps of t the difference is off by t^2 / 6 of the third derivative along the direction, and by
    fp32's errors over t; inputs are sixteenths up to 1 and the direction's entries 0 or +-1, so that
    both ends are bf16 values."""
    gen = torch.Generator(DEV).manual_seed(6)
    some = lambda r, c, top: (torch.randint(-top, top + 1, (r, c), device=DEV, generator=gen) /
                              16).bfloat16()
    m, n, k, t = 24, 40, 48, 2.0 ** -4
    at = [some(m, k, 16), some(n, k, 8), some(n, k, 8)]
    dh = some(m, n, 16)
    # relu's kinks stay out of the way: fp32's sums of these are exact, and those that a step
    # could carry over 0 take no part
    if act == "relu":
        g = at[0].double() @ at[1].double().t()
        dh = torch.where(g.abs() <= 0.25, 0.0, dh.float()).bfloat16()

    def value(sign):
        moved = [p + sign * t * ways if i == which else p for i, p in enumerate(at)]
        h = lt.gated_linear(*moved, act, out_dtype=torch.float32)
        return float((h.double() * dh.double()).sum())

    h, saved = lt.gated_linear_forward(*at, act)
    grads = lt.gated_linear_backward(dh, saved, *at, torch.float32, torch.float32)
    ways = torch.zeros_like(at[which])
    for place in ((3, 5), (7, 11), (20, 40)):  # each with its slope's sign, so that they add up
        ways[place] = torch.sign(grads[which][place])
    got = float((grads[which].double() * ways.double()).sum())
    want = (value(1) - value(-1)) / (2 * t)
    # the rows that the direction touches: their |dh| (1) times |u| (some 8) and the moves (up to 1)
    # of the others' sums; act''' is at most 1.5: n or m entries for each of three moves
    count = 3 * max(m, n)
    truncation = t * t / 6 * (1.5 * 8 + 3 * 0.8) * math.sqrt(count) * 3
    rounding = 3 * HALF * math.sqrt(count) * 8 + count * 64 * 2.0 ** -20 / t
    assert abs(got - want) <= truncation + rounding, (got, want)


def test_autograd():
    x, gate, up, dh = inputs(70, 130, 64)
    leaves = [t.clone().requires_grad_() for t in (x, gate, up)]
    lt.GatedLinear.apply(*leaves, "gelu").backward(dh)
    h, saved = lt.gated_linear_forward(x, gate, up, "gelu")
    for leaf, want in zip(leaves, lt.gated_linear_backward(dh, saved, x, gate, up)):
        assert torch.equal(leaf.grad, want)
    # one at a time, batches, the same weight twice
    for i in range(3):
        ts = [t.clone().requires_grad_(j == i) for j, t in enumerate((x.view(7, 10, 64), gate, up))]
        y = lt.GatedLinear.apply(*ts, "gelu")
        assert y.shape == (7, 10, 130)
        y.backward(dh.view(7, 10, 130))
        assert torch.equal(ts[i].grad.reshape(leaves[i].shape), leaves[i].grad)
    w = gate.clone().requires_grad_()
    lt.GatedLinear.apply(x, w, w, "relu").backward(dh)
    h, saved = lt.gated_linear_forward(x, gate, gate, "relu")
    _, a, b = lt.gated_linear_backward(dh, saved, x, gate, gate)
    assert torch.equal(w.grad, a + b)
    # broadcast tokens: their gradients add up
    one = x[:1].clone().requires_grad_()
    lt.GatedLinear.apply(one.expand(70, 64), gate, up).backward(dh)
    h, saved = lt.gated_linear_forward(x[:1].expand(70, 64), gate, up)
    dx = lt.gated_linear_backward(dh, saved, x[:1].expand(70, 64), gate, up)[0]
    assert torch.equal(one.grad, dx.sum(0, keepdim=True))
    assert not lt.GatedLinear.apply(x, gate, up).requires_grad


def test_autograd_refusals():
    x, gate, up, dh = inputs(40, 30, 20)
    ts = [t.clone().requires_grad_() for t in (x, gate, up)]
    y = lt.GatedLinear.apply(*ts)
    with pytest.raises(RuntimeError, match="first derivatives"):
        torch.autograd.grad(y.sum(), ts, create_graph=True)
    y = lt.GatedLinear.apply(*ts)
    with torch.no_grad():
        ts[1].mul_(2)
    with pytest.raises(RuntimeError, match="modified by an inplace"):
        y.sum().backward()


@pytest.mark.parametrize("mode", [torch.no_grad, torch.inference_mode])
def test_where_gradients_are_off_nothing_is_kept(mode):
    x, gate, up, _ = inputs(2048, 1024, 256)
    ts = [t.requires_grad_() for t in (x, gate, up)]
    eager = lt.GatedLinear.apply(*ts)  # a graph of the leaves, on the default stream
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with mode():
        want = lt.gated_linear(*ts, "gelu")
        torch.cuda.synchronize()
        torch.cuda.reset_peak_memory_stats()
        before = torch.cuda.memory_allocated()
        y = lt.GatedLinear.apply(*ts, "gelu")
        assert torch.cuda.max_memory_allocated() - before < 6 * 2048 * 1024
        assert torch.equal(y, want) and not y.requires_grad
        with torch.cuda.stream(side):
            with torch.cuda.graph(graph, stream=side):
                y = lt.GatedLinear.apply(*ts, "gelu")
            graph.replay()
        side.synchronize()
        assert torch.equal(y, want)
    assert eager.requires_grad


def test_layouts_and_empties():
    x, gate, up, dh = inputs(48, 130, 70)
    h, saved = lt.gated_linear_forward(x, gate, up)
    grads = lt.gated_linear_backward(dh, saved, x, gate, up)
    turn = lambda t: t.t().contiguous().t()

    def wide(t, at):
        big = torch.full((t.shape[0], t.shape[1] + 13), float("nan"), device=DEV).to(t.dtype)
        big[:, at:at + t.shape[1]] = t
        return big[:, at:at + t.shape[1]]

    for change in (turn, lambda t: wide(t, 0), lambda t: wide(t, 8), lambda t: wide(t, 5)):
        ts = [change(t) for t in (x, gate, up)]
        assert torch.equal(lt.gated_linear(*ts), lt.gated_linear(x, gate, up))
        h2, saved2 = lt.gated_linear_forward(*ts)
        assert torch.equal(h2, h)
        for a, b in zip(lt.gated_linear_backward(change(dh), saved2, *ts), grads):
            assert torch.equal(a, b)
    both = torch.cat([gate, up])           # one matrix holds both
    assert torch.equal(lt.gated_linear(x, both[:130], both[130:]), lt.gated_linear(x, gate, up))
    assert torch.equal(lt.gated_linear(x.view(2, 24, 70), gate, up).view(48, 130),
                       lt.gated_linear(x, gate, up))
    assert torch.equal(lt.gated_linear(x[5], gate, up), lt.gated_linear(x[5:6], gate, up)[0])

    for m, n, k in [(0, 130, 70), (48, 0, 70), (48, 130, 0), (0, 0, 0)]:
        a, b, c, d = x[:m, :k], gate[:n, :k], up[:n, :k], dh[:m, :n]
        h, saved = lt.gated_linear_forward(a, b, c)
        assert h.shape == (m, n) and not h.any()
        assert lt.gated_linear(a, b, c).shape == (m, n)
        dx, dg, du = lt.gated_linear_backward(d, saved, a, b, c)
        assert dx.shape == (m, k) and dg.shape == du.shape == (n, k)
        assert not dx.any() and not dg.any() and not du.any()


def test_bad_tokens_stay_alone():
    """A NaN or an infinity in a token reaches its own row, and the weights' gradients in the
    places that read it: columns of x with it, rows of channels without bounds."""
    for m in (20, 200):
        x, gate, up, dh = inputs(m, 96, 130)
        h0, saved0 = lt.gated_linear_forward(x, gate, up)
        dx0, _, _ = lt.gated_linear_backward(dh, saved0, x, gate, up)
        y0 = lt.gated_linear(x, gate, up)
        x = x.clone()
        x[m - 1, 129] = float("nan")
        h, saved = lt.gated_linear_forward(x, gate, up)
        dx, dg, du = lt.gated_linear_backward(dh, saved, x, gate, up)
        y = lt.gated_linear(x, gate, up)
        for got, want in ((h, h0), (dx, dx0), (y, y0)):
            assert torch.isnan(got[m - 1]).all() and torch.equal(got[:m - 1], want[:m - 1])
        assert torch.isnan(dg).all() and torch.isnan(du).all()
        # a gradient that is not finite
        d = dh.clone()
        d[3, 5] = float("inf")
        h, saved = lt.gated_linear_forward(x[:19], gate, up)
        dx, dg, du = lt.gated_linear_backward(d[:19], saved, x[:19], gate, up)
        fine = torch.isfinite(dx).all(1)
        assert not fine[3] and int(fine.sum()) == 18
        fine = torch.isfinite(dg).all(1)
        assert not fine[5] and int(fine.sum()) == 95


def test_saved_is_a_program_s_to_keep():
    """Two forward passes before either backward, in either order."""
    a, b = inputs(70, 96, 64), inputs(40, 96, 64)
    fa, fb = lt.gated_linear_forward(*a[:3]), lt.gated_linear_forward(*b[:3], "relu")
    gb = lt.gated_linear_backward(b[3], fb[1], *b[:3])
    ga = lt.gated_linear_backward(a[3], fa[1], *a[:3])
    fa, fb = lt.gated_linear_forward(*a[:3]), lt.gated_linear_forward(*b[:3], "relu")
    for x, y in zip(ga + gb, lt.gated_linear_backward(a[3], fa[1], *a[:3]) +
                    lt.gated_linear_backward(b[3], fb[1], *b[:3])):
        assert torch.equal(x, y)
