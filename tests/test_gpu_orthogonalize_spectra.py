"""The tiled ways of lt_orthogonalize on steep spectra: singular values over decades, one or a few
directions far above the rest, directions that are missing.

Tolerances come from a model of the roundings, evaluated in 64 bits for every input: X and every
n x n matrix that a way stores (header of csrc/orth.hip: S, P, W, S', P', R and X's leading half,
without their multiples of I) is off by an independent relative error of up to 2^-11, fp16's, in
every element, uniformly drawn; the sum of X's two halves by 2^-22.  Nothing else rounds to fewer
than 24 bits.  The model's distance from the polynomial is what the roundings make of this
input, whatever their signs; uniform errors of the largest relative size are some 1.4 times those
of rounding, and the tolerance is twice the larger of two draws."""
import pytest
import torch

import paper_2608_11919_amd as lt

pytestmark = pytest.mark.gpu
DEV = "cuda"
A, B, C = 3.4445, -4.7750, 2.0315
F64 = torch.float64


def exact(u, steps=5):
    x = u / torch.linalg.vector_norm(u)
    for _ in range(steps):
        g = x @ x.t()
        x = A * x + (B * g + C * (g @ g)) @ x
    return x


def modelled(u, pairs, gen, steps=5):
    """The steps on u (rows its smaller side) with a random error wherever fp16 stores."""
    def off(x, eps=2.0 ** -11):
        return x * (1 + eps * (2 * torch.rand(x.shape, dtype=F64, device=DEV, generator=gen) - 1))

    n = u.shape[0]
    eye = torch.eye(n, dtype=F64, device=DEV)
    x, d, step = u / torch.linalg.vector_norm(u), 1.0 / n, 0
    while step < steps:
        head, x = off(x), off(x, 2.0 ** -22)
        p = A + d * (B + C * d)
        s = off(head @ head.t() - d * eye)
        ph = off(C * s @ s + (B + 2 * C * d) * s)
        if pairs and step + 1 < steps:
            w = off(ph @ s + p * s + d * ph)
            s2 = off(ph @ w + p * w + p * d * ph)
            d2 = p * p * d
            p2 = A + d2 * (B + C * d2)
            ph2 = off(C * s2 @ s2 + (B + 2 * C * d2) * s2)
            r = off(ph2 @ ph + p2 * ph + p * ph2)
            x = p2 * p * x + r @ head
            d, step = p2 * p2 * d2, step + 2
        else:
            x = p * x + ph @ head
            d, step = p * p * d, step + 1
    return x


def with_values(n, m, values, gen):
    """A matrix of n <= m rows with these singular values."""
    q, _ = torch.linalg.qr(torch.randn(n, n, dtype=F64, device=DEV, generator=gen))
    r, _ = torch.linalg.qr(torch.randn(m, n, dtype=F64, device=DEV, generator=gen))
    return (q * values) @ r.t()


def decades(k):
    return lambda n, m, g: with_values(n, m, 10.0 ** (-k * torch.linspace(0, 1, n, dtype=F64,
                                                                          device=DEV)), g)


def directions(k, factor):
    def make(n, m, g):
        values = torch.ones(n, dtype=F64, device=DEV)
        values[:k] = factor
        return with_values(n, m, values, g)
    return make


def noise(*shape, g):
    return torch.randn(*shape, dtype=F64, device=DEV, generator=g)


SPECTRA = {
    "noise": lambda n, m, g: noise(n, m, g=g),
    "flat": decades(0), "1 decade": decades(1), "3 decades": decades(3), "4 decades": decades(4),
    "6 decades": decades(6),
    "2 directions 100 above": directions(2, 1e2), "8 directions 1000 above": directions(8, 1e3),
    "1 direction 10000 above": directions(1, 1e4),
    "1 direction far above noise": lambda n, m, g: noise(n, m, g=g) +
    1e3 * noise(n, 1, g=g) @ noise(1, m, g=g),
    "rank 1": lambda n, m, g: noise(n, 1, g=g) @ noise(1, m, g=g),
    "half the rank": lambda n, m, g: noise(n, n // 2, g=g) @ noise(n // 2, m, g=g),
    "rows of scales 1 to 0.01": lambda n, m, g: noise(n, m, g=g) *
    10.0 ** (-2 * torch.linspace(0, 1, n, dtype=F64, device=DEV))[:, None],
    "rows of zeros": lambda n, m, g: noise(n, m, g=g) *
    (torch.arange(n, device=DEV) % 3 == 0)[:, None],
}
# smaller and longer side: the first four in single steps, the others in pairs
SIDES = [(65, 300), (100, 150), (200, 200), (500, 600), (128, 256), (130, 2000), (300, 700),
         (512, 2048)]


@pytest.mark.parametrize("tall", [False, True])
@pytest.mark.parametrize("sides", SIDES, ids=str)
@pytest.mark.parametrize("spectrum", SPECTRA)
def test_spectrum(spectrum, sides, tall):
    n, m = sides
    gen = torch.Generator(DEV).manual_seed(n + m)
    u = SPECTRA[spectrum](n, m, gen)
    u = (u / u.abs().max()).float()
    given = u.t().contiguous() if tall else u
    out = torch.empty_like(given)
    lt.lt_orthogonalize([given], [out])
    got = (out.t() if tall else out).double()
    want = exact(u.double())
    size = torch.linalg.vector_norm(want).item()
    pairs = n >= 128 and m >= 2 * n
    model = [torch.linalg.vector_norm(modelled(u.double(), pairs, gen) - want).item() / size
             for _ in range(2)]
    off = torch.linalg.vector_norm(got - want).item() / size
    print(f"off {off:.2e} model {max(model):.2e} {'pairs' if pairs else 'single'} {n} x {m} "
          f"{spectrum}")
    assert off <= 2 * max(model)
