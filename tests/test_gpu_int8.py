"""8-bit integer quantizer, products and layers on the GPU.

Everything but the activations is bitwise.  A code is the nearest integer to x times one fp32
quotient, whose exact product fits 64 bits; a sum of codes' products is an integer; what follows is
three roundings of fp32, which numpy makes alike, and one to the result's type."""
import numpy as np
import pytest
import torch

import paper_2608_11919_amd as lt

pytestmark = pytest.mark.gpu
DEV = "cuda"


def expected(x):
    """Codes and scales of x, a torch matrix, by the definition in 64 bits."""
    v = x.double().cpu().numpy()
    most = np.abs(v).max(1, initial=0.0)
    bad = ~np.isfinite(most)
    most32 = np.maximum(np.where(bad, 1.0, most), 2.0 ** -100).astype(np.float32)
    factor, scale = np.float32(127) / most32, most32 / np.float32(127)
    with np.errstate(invalid="ignore"):
        codes = np.rint(v * factor.astype(np.float64)[:, None])
    codes[bad] = 0
    return codes.astype(np.int64), np.where(bad, np.float32(np.nan), scale)


def quantize(x):
    rows, cols = x.shape
    codes = torch.full((rows, lt.lt_int8_code_pitch(cols)), 99, dtype=torch.int8, device=DEV)
    scales = torch.full((rows,), 7.0, device=DEV)
    lt.lt_int8_quantize(x, codes, scales)
    return codes, scales


def matrix(rows, cols, seed, dtype, spread=True):
    gen = torch.Generator(DEV).manual_seed(seed)
    x = torch.randn(rows, cols, device=DEV, generator=gen)
    if spread:
        x = x * torch.exp(3 * torch.randn(rows, 1, device=DEV, generator=gen))
    return x.to(dtype)


def check_codes(x):
    codes, scales = quantize(x)
    want, s = expected(x)
    assert np.array_equal(scales.cpu().numpy(), s, equal_nan=True)
    got = codes.cpu().numpy().astype(np.int64)
    assert np.array_equal(got[:, :x.shape[1]], want)
    assert not got[:, x.shape[1]:].any()


@pytest.mark.parametrize("shape", [(1, 1), (3, 7), (5, 128), (129, 127), (6, 513), (300, 2048),
                                   (3, 2049), (9, 4100), (2, 8192), (3, 20001)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_quantizer(shape, dtype):
    check_codes(matrix(*shape, 3, dtype))


@pytest.mark.parametrize("cols", [40, 700, 3000, 9000])
def test_quantizer_edges(cols):
    """Rows of zeros, of the least and largest numbers, of ties, with a NaN or an infinity; views
    that begin at any element."""
    x = matrix(12, cols + 3, 5, torch.float32)[:, 3:]
    x[0] = 0.0
    x[1] *= 1e-44
    x[2] = torch.where(x[2] > 0, 3.4028234e38, -1e37)
    x[3, cols // 2] = float("nan")
    x[4, cols - 1] = float("-inf")
    x[5] = torch.arange(cols, device=DEV) % 128 - 63.5     # most / 2 lies between two codes
    x[5, 0] = 127.0
    x[6] = 2.0 ** -101
    x[7] = -0.0
    x[8, :] = -1.0
    check_codes(x)
    check_codes(x.bfloat16())
    check_codes(x.bfloat16()[:, 1:])


def product(a, b, dtype):
    """Bits of the product by the definition; a, b are (codes, scales) from expected()."""
    sums = a[0] @ b[0].T
    with np.errstate(invalid="ignore", over="ignore"):
        y = sums.astype(np.float32) * a[1][:, None] * b[1][None, :]
    return torch.from_numpy(y).to(dtype)


def same(got, want):
    want = want.to(got.device)
    return torch.equal(torch.isnan(got), torch.isnan(want)) and \
        torch.equal(got.nan_to_num(0.0), want.nan_to_num(0.0))


SIZES = [(1, 1, 1), (1, 520, 300), (2, 17, 129), (16, 33, 1000), (17, 300, 128), (32, 64, 2048),
         (5, 9000, 2048), (16, 8300, 2049), (3, 4200, 5121), (16, 70, 8192), (2, 70, 8193),
         (33, 65, 127), (64, 64, 6400), (65, 200, 9001), (100, 1, 12800), (300, 257, 257),
         (129, 4096, 640), (520, 2050, 96), (1030, 16390, 130), (1, 300, 17000), (16, 1, 20001)]


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_products(m, n, k, dtype):
    a, b = matrix(m, k, 1, torch.float32), matrix(n, k, 2, torch.bfloat16)
    ca, cb = quantize(a), quantize(b)
    wide = torch.full((m, n + 5), 5.0, dtype=dtype, device=DEV)
    out = wide[:, :n]
    lt.lt_int8_matmul(*ca, *cb, k, out)
    want = product(expected(a), expected(b), dtype)
    assert same(out, want)
    assert (wide[:, n:] == 5.0).all()
    # the layer quantizes a itself: the same bits
    y = lt.int8_linear(a, lt.Int8Weight.from_master(b), out_dtype=dtype)
    assert same(y, want)


def test_largest_sum():
    """2^17 products of the largest codes fit the accumulators."""
    k = 1 << 17
    for m in (1, 40):
        a = torch.full((m, k), 127, dtype=torch.int8, device=DEV)
        b = torch.full((3, k), -127, dtype=torch.int8, device=DEV)
        out = torch.empty(m, 3, device=DEV)
        one = lambda n: torch.ones(n, device=DEV)
        lt.lt_int8_matmul(a, one(m), b, one(3), k, out)
        assert (out == -float(127 * 127 * k)).all()


@pytest.mark.parametrize("m", [2, 20, 70, 600])
def test_a_bad_token_stays_alone(m):
    x, w = matrix(m, 300, 1, torch.bfloat16), matrix(200, 300, 2, torch.float32)
    w[7, 3] = float("inf")
    x[1, 5] = float("nan")
    y = lt.int8_linear(x, lt.Int8Weight.from_master(w))
    assert same(y, product(expected(x), expected(w), torch.bfloat16))
    bad = torch.isnan(y)
    assert bad[1].all() and bad[:, 7].all() and int(bad.sum()) == m + 200 - 1


@pytest.mark.parametrize("m", [3, 90])
def test_a_bad_token_of_a_long_sum_stays_alone(m):
    x = matrix(m, 9000, 1, torch.bfloat16)
    ws = [lt.Int8Weight.from_master(matrix(70, 9000, s, torch.float32)) for s in (2, 3)]
    want = lt.int8_gated_linear(x, *ws)
    assert torch.isfinite(want).all()
    x[2, 8999] = float("inf")
    got = lt.int8_gated_linear(x, *ws)
    assert torch.isnan(got[2]).all()
    assert torch.equal(got[:2], want[:2]) and torch.equal(got[3:], want[3:])


def test_layouts_and_empties():
    w = lt.Int8Weight.from_master(matrix(130, 70, 2, torch.float32))
    x = matrix(24, 70, 1, torch.bfloat16)
    want = lt.int8_linear(x, w)
    assert torch.equal(lt.int8_linear(x.view(2, 3, 4, 70), w), want.view(2, 3, 4, 130))
    assert torch.equal(lt.int8_linear(x[3], w), want[3])
    assert torch.equal(lt.int8_linear(x.t().contiguous().t(), w), want)
    wide = torch.zeros(24, 99, dtype=torch.bfloat16, device=DEV)
    wide[:, 11:81] = x
    assert torch.equal(lt.int8_linear(wide[:, 11:81], w), want)
    assert torch.equal(lt.int8_linear(x[2:3].expand(5, 70), w), want[2:3].expand(5, 130))
    assert lt.int8_linear(x[:0], w).shape == (0, 130)
    assert lt.int8_linear(x.view(6, 4, 70)[:, :0], w).shape == (6, 0, 130)
    none = lt.Int8Weight.from_master(torch.empty(130, 0, device=DEV))
    assert (lt.int8_linear(x[:, :0], none) == 0).all()
    no_rows = lt.Int8Weight.from_master(torch.empty(0, 70, device=DEV))
    assert lt.int8_linear(x, no_rows).shape == (24, 0)
    turned = lt.Int8Weight.from_master(matrix(70, 130, 3, torch.float32).t())
    assert torch.equal(turned.codes, lt.Int8Weight.from_master(
        matrix(70, 130, 3, torch.float32).t().contiguous()).codes)


# The activation of the fp32 product g and its product with u, against 64 bits.  g and u are three
# roundings off the exact ones, 3 * 2^-24.  e^-z comes from a product with log2(e) (1.5 * 2^-24 |z|
# of the result), a power of two (2^-23), a sum (2^-24) and a reciprocal (2^-23); act(g) moves by
# |g act'(g) / act(g)| as much, relatively, as g does: at most 1 + |g| for silu, 1 + 3 |z| for
# gelu_tanh with z = g (c + d g^2), itself three roundings off, and 1 + g^2 for gelu, whose
# e^(-g^2/2) has an argument 2.5 * 2^-24 off, too (1.25 g^2 of the result), and whose polynomial is
# some 15 * 2^-24 off itself.
ROOM = {"silu": lambda g: 5 * abs(g) + 20, "relu": lambda g: 12 + 0 * g,
        "gelu_tanh": lambda g: 15 * abs(g * (1.6 + 0.072 * g * g)) + 24,
        "gelu": lambda g: 8 * g * g + 40}


def activation(name, g):
    if name == "silu":
        return g * torch.sigmoid(g)
    if name == "gelu":
        return 0.5 * g * torch.special.erfc(-g * 0.5 ** 0.5)
    if name == "gelu_tanh":
        return g * torch.sigmoid(2 * (2 / torch.pi) ** 0.5 * (g + 0.044715 * g ** 3))
    return g.clamp_min(0)


@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 520, 300), (16, 33, 1000), (17, 300, 128),
                                   (16, 9000, 700), (5, 4200, 2100), (3, 300, 8000), (2, 40, 8300),
                                   (33, 65, 127), (65, 200, 3001), (300, 257, 257),
                                   (129, 4096, 640), (520, 2050, 96), (1030, 8200, 130),
                                   (1, 70, 17000), (40, 70, 4096), (300, 130, 9001)])
@pytest.mark.parametrize("act", list(ROOM))
def test_gated(m, n, k, act):
    x = matrix(m, k, 1, torch.bfloat16, spread=False)
    ws = [matrix(n, k, s, torch.float32, spread=False) * (2 / k ** 0.5) for s in (2, 3)]
    gate, up = (lt.Int8Weight.from_master(w) for w in ws)
    g, u = (torch.from_numpy(q[0] @ p[0].T * (q[1].astype(np.float64)[:, None] *
                                              p[1].astype(np.float64)[None, :]))
            for q in [expected(x)] for p in map(expected, ws))
    a = activation(act, g)
    want = a * u
    for dtype in (torch.float32, torch.bfloat16):
        got = lt.int8_gated_linear(x, gate, up, act, out_dtype=dtype).double().cpu()
        room = ROOM[act](g) * 2.0 ** -24 + torch.finfo(dtype).eps / 2
        assert ((got - want).abs() <= room * want.abs() + 1e-36).all(), \
            ((got - want).abs() / want.abs()).max()


def test_gated_takes_any_layout():
    gate, up = (lt.Int8Weight.from_master(matrix(130, 70, s, torch.float32)) for s in (2, 3))
    x = matrix(48, 70, 1, torch.float32)
    want = lt.int8_gated_linear(x, gate, up, "gelu")
    assert torch.equal(lt.int8_gated_linear(x.view(2, 24, 70), gate, up, "gelu"),
                       want.view(2, 24, 130))
    assert torch.equal(lt.int8_gated_linear(x.t().contiguous().t(), gate, up, "gelu"), want)
    assert lt.int8_gated_linear(x[:0], gate, up).shape == (0, 130)
    none = lt.Int8Weight.from_master(torch.empty(130, 0, device=DEV))
    assert (lt.int8_gated_linear(x[:, :0], none, none) == 0).all()
