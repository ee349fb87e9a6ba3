"""Matrices with a small side of 1 to 64, short and long, against the definition in 64 bits.

Their Gram matrix and steps are in 64 bits, where an error grows to 1e-9 of R at most; R is rounded
to fp32 once and R X0 summed in fp32 over up to 64 terms, one scale factor on each side:
    |got - exact| <= ((n + 8) 2^-24 + 1e-8) (|R| |X0|) + half a unit of the output type,
every element for itself."""
import pytest
import torch

import paper_2608_11919_amd as lt

pytestmark = pytest.mark.gpu
DEV = "cuda"
A, B, C = 3.4445, -4.7750, 2.0315
SIDES = [(1, 1), (1, 5000), (3, 129), (16, 2049), (17, 511), (31, 4097), (32, 4288), (32, 9000),
         (33, 33), (33, 1025), (48, 100), (63, 64), (64, 64), (64, 513), (64, 2048), (50, 5003)]


def exact(u, steps):
    """(result, bound without the output's rounding) of one matrix, both float64."""
    x = u.double()
    tall = x.shape[0] > x.shape[1]
    x = x.t() if tall else x
    n = x.shape[0]
    norm = x.norm()
    x0 = x / norm if norm > 0 else x
    g, eye = x0 @ x0.t(), torch.eye(n, dtype=torch.float64, device=x.device)
    r = eye
    for _ in range(steps):
        p = A * eye + B * g + C * g @ g
        r, g = p @ r, p @ g @ p
    o = r @ x0
    bound = ((n + 8) * 2.0 ** -24 + 1e-8) * (r.abs() @ x0.abs())
    return (o.t(), bound.t()) if tall else (o, bound)


def check(got, u, steps=5):
    o, bound = exact(u, steps)
    half = 2.0 ** -8 if got.dtype == torch.bfloat16 else 2.0 ** -24  # 8 and 24 significant bits
    bound = bound + half * (o.abs() + bound) + 1e-38
    worst = ((got.double() - o).abs() / bound).max().item()
    assert worst <= 1.0, worst


def draw(rows, cols, seed, kind="noise"):
    gen = torch.Generator(DEV).manual_seed(seed)
    u = torch.randn(rows, cols, device=DEV, generator=gen)
    if kind == "rows":  # rows (or columns) of scales from 1 to 0.01
        n = min(rows, cols)
        scale = 10.0 ** (-2.0 * torch.arange(n, device=DEV) / max(n - 1, 1))
        u = u * (scale[:, None] if rows <= cols else scale[None, :])
    return u


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind", ["noise", "rows"])
@pytest.mark.parametrize("tall", [False, True])
@pytest.mark.parametrize("side", SIDES, ids=str)
def test_one_matrix(side, tall, kind, dtype):
    shape = side[::-1] if tall else side
    u = draw(*shape, 1, kind).to(dtype)
    out = torch.empty(shape, device=DEV, dtype=dtype)
    lt.lt_orthogonalize([u], [out])
    check(out, u.float())


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("steps", [1, 2, 7])
def test_many_of_all_kinds(steps, out_dtype):
    shapes = [s if i % 2 else s[::-1] for i, s in enumerate(SIDES)] * 20  # more than CUs
    us = [draw(*s, i) for i, s in enumerate(shapes)]
    out = [torch.empty(s, device=DEV, dtype=out_dtype) for s in shapes]
    lt.lt_orthogonalize(us, out, ns_steps=steps)
    for o, u in zip(out[:len(SIDES)] + out[-3:], us[:len(SIDES)] + us[-3:]):
        check(o, u, steps)
    again = [torch.empty_like(o) for o in out]
    lt.lt_orthogonalize(us, again, ns_steps=steps)
    assert all(torch.equal(a, b) for a, b in zip(out, again))


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("shape", [(64, 700), (700, 40)])
def test_zero_and_nan_keep_to_their_matrix(shape, value):
    bad, zero, good = draw(*shape, 1), torch.zeros(shape, device=DEV), draw(*shape, 2)
    bad[3, 5] = value
    out = [torch.full(shape, 7.0, device=DEV) for _ in range(3)]
    lt.lt_orthogonalize([bad, zero, good], out)
    assert out[0].isnan().all() and (out[1] == 0).all()
    check(out[2], good)


@pytest.mark.parametrize("scale", [1e-30, 1e-15, 1e15, 1e30])
def test_scale_does_not_matter(scale):
    u = draw(64, 900, 3)
    out = torch.empty_like(u)
    lt.lt_orthogonalize([u * scale], [out])
    check(out, u * scale)


@pytest.mark.parametrize("shape", [(32, 4288), (4288, 32), (64, 1030), (1030, 64), (1, 600), (45, 45)])
@pytest.mark.parametrize("copy", [False, True])
def test_muon_step(shape, copy):
    """momentum 0: the update is the gradient itself."""
    w0, g = draw(*shape, 5), draw(*shape, 6)
    w = w0.clone()
    n = w.numel()
    codes = torch.zeros(n, dtype=torch.int8, device=DEV)
    absmax = torch.zeros(-(-n // 256), device=DEV)
    wb = torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    status = torch.ones(1, dtype=torch.int32, device=DEV)
    hyper = dict(lr=0.01, momentum=0.0, nesterov=False, weight_decay=0.1, update_rms=0.2,
                 status=status, params_bf16=[wb] if copy else None)
    lt.lt_muon_step([w], [g], [codes], [absmax], 256, **hyper)
    assert torch.equal(w, w0) and (codes == 0).all()  # skipped
    if copy:
        assert torch.equal(wb, w0.view(-1).bfloat16())
    status.zero_()
    lt.lt_muon_step([w], [g], [codes], [absmax], 256, **hyper)
    o, bound = exact(g, 5)
    rate = 0.01 * 0.2 * max(shape) ** 0.5
    want = w0.double() * (1 - 0.01 * 0.1) - rate * o
    limit = rate * (bound + 2.0 ** -22 * o.abs()) + 2.0 ** -22 * (w0.double().abs() + want.abs())
    assert ((w.double() - want).abs() <= limit).all()
    if copy:
        assert torch.equal(wb, w.view(-1).bfloat16())
