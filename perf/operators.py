"""The matrix operators of a training program, as cases a measuring program can run.

Three kinds of pass, through the public entry points of ``paper_2608_11919_amd``:

* ``orth``: the Newton-Schulz orthogonalisation of a list of matrices;
* ``muon``: the clipped Muon step with 8-bit momentum that is built on it;
* ``linear`` and ``train``: a linear layer in 8-bit floating point with a scale for each
  block of 128, forward for serving, and forward and backward (with the weight's
  quantisation) for training.

Where ``own`` is false, ``run`` computes the same in elementary torch operations in 32
bits.  ``exact`` restates the definitions in 64 bits.  Matrices of one shape are held as
one stack, so that outputs are a handful of tensors however many matrices a list has.
"""
import math
import random

import torch

own = False

A, B, C = 3.4445, -4.7750, 2.0315     # coefficients of the Newton-Schulz polynomial
NS_STEPS = 5
LR, MOMENTUM, WEIGHT_DECAY, UPDATE_RMS = 2e-5, 0.95, 0.01, 0.2
COEF = 0.5                            # a clip coefficient as a clipped step has it
GROUP = 128                           # elements that share a scale in 8-bit floating point


# ---------------------------------------------------------------------- cases

def listed():
    return [
        # Low-rank adapters (rank 16) on the four projections of one layer of the
        # 3B-class model: eight thin matrices, the smallest call.
        dict(name="orth_adapter_layer", op="orth", kind="adapters", layers=1, hidden=2048, rank=16,
             dtype="f32"),
        # Matrices of odd sizes from a single element to a thousand rows.
        dict(name="orth_odd", op="orth", kind="odd", sizes=7, count=8, largest=1500, dtype="bf16"),
        # The projections of one layer of the 3B-class model, bf16 momentum.
        dict(name="orth_layer_3b", op="orth", kind="decoder", hidden=2048, ffn=11008, kv=256,
             dtype="bf16"),
        # One feed-forward matrix of the 27B-class model, fp32 momentum.
        dict(name="orth_ffn_27b", op="orth", kind="one", rows=17408, cols=5120, dtype="f32"),
        # The whole adapter set of 36 layers (288 matrices) in one step, dynamic codes.
        dict(name="muon_adapters", op="muon", kind="adapters", layers=36, hidden=2048, rank=16,
             block=512, map="dynamic", dtype="bf16", copy=False),
        # One decoder layer of the 3B-class model: bf16 gradients, the paper's block size,
        # and the bf16 copy for the next forward pass.
        dict(name="muon_layer_3b", op="muon", kind="decoder", hidden=2048, ffn=11008, kv=256,
             block=4096, map="linear", dtype="bf16", copy=True),
        # One decoder layer of the 27B-class model with fp32 gradients: the largest step.
        dict(name="muon_layer_27b", op="muon", kind="decoder", hidden=5120, ffn=17408, kv=1024,
             block=2048, map="linear", dtype="f32", copy=False),
        # A single token through a feed-forward matrix of the 3B-class model.
        dict(name="linear_one_token", op="linear", tokens=1, cols=2048, rows=11008, dtype="bf16"),
        # Sixteen sequences answering at once, 27B-class feed-forward matrix.
        dict(name="linear_16_tokens", op="linear", tokens=16, cols=5120, rows=17408, dtype="bf16"),
        # A ragged prompt through a layer whose sizes are no multiples of anything.
        dict(name="linear_ragged_prompt", op="linear", tokens=1237, cols=2011, rows=5003,
             dtype="f32"),
        # Forward and backward of 8192 tokens (eight sequences of 1024, the paper's length),
        # 3B-class feed-forward matrix.
        dict(name="train_ffn_3b", op="train", tokens=8192, cols=2048, rows=11008, dtype="bf16"),
        # The same at twice the tokens on the 27B-class feed-forward matrix.
        dict(name="train_ffn_27b", op="train", tokens=16384, cols=5120, rows=17408, dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed kinds, over their whole ranges."""
    op = rng.choice(["orth", "muon", "linear", "linear", "train"])
    if op in ("orth", "muon"):
        kind = rng.choice(["adapters", "odd", "decoder", "decoder", "one"])
        c = dict(op=op, kind=kind, dtype=rng.choice(["bf16", "f32"]))
        if kind == "adapters":
            c.update(layers=rng.randint(1, 40), hidden=64 * rng.randint(8, 80),
                     rank=rng.choice([4, 8, 16, 32, 64]))
        elif kind == "odd":
            c.update(sizes=rng.randrange(1 << 20), count=rng.randint(2, 14),
                     largest=_log_int(rng, 40, 4000))
        elif kind == "decoder":
            hidden = 64 * _log_int(rng, 4, 64)
            c.update(hidden=hidden, ffn=hidden * rng.randint(8, 20) // 4 | rng.randint(0, 1),
                     kv=64 * rng.randint(1, hidden // 64))
        else:
            c.update(rows=_log_int(rng, 64, 17408), cols=_log_int(rng, 64, 5120))
        if op == "muon":
            c.update(block=rng.choice([64, 192, 256, 512, 768, 1024, 2048, 4096, 8192, 16384]),
                     map=rng.choice(["linear", "dynamic"]), copy=rng.random() < 0.5)
        return c
    c = dict(op=op, dtype=rng.choice(["bf16", "bf16", "f32"]), cols=_log_int(rng, 64, 5120),
             rows=_log_int(rng, 64, 17408))
    if rng.random() < 0.6:      # model dimensions are mostly multiples of 64
        c["cols"], c["rows"] = -(-c["cols"] // 64) * 64, -(-c["rows"] // 64) * 64
    c["tokens"] = _log_int(rng, 1, 4096) if op == "linear" else _log_int(rng, 64, 12288)
    return c


def _groups(case):
    """[(count, rows, cols)]: the matrices of a list, by shape."""
    if case["kind"] == "adapters":
        n = 4 * case["layers"]
        return [(n, case["rank"], case["hidden"]), (n, case["hidden"], case["rank"])]
    if case["kind"] == "odd":
        r = random.Random(case["sizes"])
        return [(1, 1, 1), (1, 1, case["largest"])] + \
            [(1, _log_int(r, 1, case["largest"]), _log_int(r, 1, case["largest"]))
             for _ in range(case["count"])]    # odd sizes: every matrix its own allocation
    if case["kind"] == "one":
        return [(1, case["rows"], case["cols"])]
    h, f, kv = case["hidden"], case["ffn"], case["kv"]
    return [(2, h, h), (2, kv, h), (2, f, h), (1, h, f)]


# ---------------------------------------------------------------------- inputs

_DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


def _gradients(count, rows, cols, gen, dtype):
    """Gradients as a batch of tokens leaves them: a few strong directions over noise."""
    dev = "cuda"
    k = max(1, min(rows, cols, 32) // 2)
    strength = torch.arange(1, k + 1, device=dev, dtype=torch.float32).reciprocal()
    left = torch.randn(count, rows, k, device=dev, generator=gen) * strength
    right = torch.randn(count, k, cols, device=dev, generator=gen)
    noise = torch.randn(count, rows, cols, device=dev, generator=gen)
    return ((torch.bmm(left, right) * 0.5 + noise) * 1e-3).to(dtype)


def _rowwise(x):
    """Quantises x [R, K] to 8-bit floating point in groups of 128 along K: codes
    [R, K up to a multiple of 128] (bytes of float8_e4m3fn) and the exponents of the
    power-of-two scales, biased by 127, [R, groups up to a multiple of 4]."""
    rows, k = x.shape
    groups = -(-k // GROUP)
    g = torch.nn.functional.pad(x.float(), (0, groups * GROUP - k)).view(rows, groups, GROUP)
    e = _exponent(g.abs().amax(-1))
    codes = (g * _power(-e).unsqueeze(-1)).to(torch.float8_e4m3fn).view(rows, groups * GROUP)
    return codes.view(torch.uint8), _biased(e, groups)


def _square(w):
    """Quantises w [N, K] with one scale for each 128 x 128 block; codes and exponents as
    _rowwise gives them, every row with those of its block."""
    n, k = w.shape
    bn, bk = -(-n // GROUP), -(-k // GROUP)
    g = torch.nn.functional.pad(w.float(), (0, bk * GROUP - k, 0, bn * GROUP - n))
    e = _exponent(g.view(bn, GROUP, bk, GROUP).abs().amax((1, 3)))
    e = e.repeat_interleave(GROUP, 0)[:n]
    codes = (g[:n].view(n, bk, GROUP) * _power(-e).unsqueeze(-1)).to(torch.float8_e4m3fn)
    return codes.view(n, bk * GROUP).view(torch.uint8), _biased(e, bk)


def _exponent(amax):
    """The least e with amax <= 448 * 2^e, and at least -126; 0 where amax is 0."""
    m, e = torch.frexp(amax)            # amax = m * 2^e, 1/2 <= m < 1; 448 = 0.875 * 2^9
    e = torch.where(m <= 0.875, e - 9, e - 8).clamp_min(-126)
    return torch.where(amax > 0, e, torch.zeros_like(e))


def _power(e):
    return ((e + 127) << 23).view(torch.float32)


def _biased(e, groups):
    return torch.nn.functional.pad((e + 127).to(torch.uint8), (0, -groups % 4), value=127)


def _values(codes, scales, k):
    """The 32-bit values that codes and exponents stand for, [R, k]."""
    rows, wide = codes.shape
    e = scales[:, :wide // GROUP].to(torch.int32) - 127
    v = codes.view(torch.float8_e4m3fn).float().view(rows, wide // GROUP, GROUP)
    return (v * _power(e).unsqueeze(-1)).view(rows, wide)[:, :k]


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    dtype = _DTYPE[case["dtype"]]
    s = dict(case=case)
    if case["op"] in ("orth", "muon"):
        groups = _groups(case)
        s["grads"] = [_gradients(n, r, c, gen, dtype) for n, r, c in groups]
        if case["op"] == "orth":
            s["out"] = [torch.empty(n, r, c, device="cuda", dtype=torch.bfloat16)
                        for n, r, c in groups]
        else:
            block = case["block"]
            s["w"] = [torch.randn(n, r, c, device="cuda", generator=gen) * 0.02
                      for n, r, c in groups]
            top = 256 if case["map"] == "dynamic" else 255
            s["codes"] = [(torch.randint(0, top, (n, r * c), device="cuda", generator=gen) -
                           (128 if top == 256 else 127)).to(torch.int8) for n, r, c in groups]
            s["absmax"] = [torch.rand(n, -(-r * c // block), device="cuda", generator=gen) * 4e-3 +
                           1e-3 for n, r, c in groups]
            s["copy"] = [torch.zeros(n, r, c, device="cuda", dtype=torch.bfloat16)
                         for n, r, c in groups] if case["copy"] else None
            s["coef"] = torch.full((1,), COEF, device="cuda")
            s["status"] = torch.zeros(1, device="cuda", dtype=torch.int32)
            s["table"] = _dynamic_table().to("cuda")
        return s
    t, k, n = case["tokens"], case["cols"], case["rows"]
    s["x"] = torch.randn(t, k, device="cuda", generator=gen).to(dtype)
    w = torch.randn(n, k, device="cuda", generator=gen) / math.sqrt(k)
    if case["op"] == "linear":
        s["wq"], s["ws"] = _square(w)   # laid out once, kept by the program
    else:
        s["w"] = w                      # the master weights that the optimizer updates
        s["dy"] = (torch.randn(t, n, device="cuda", generator=gen) * 1e-3).to(dtype)
    return s


# ---------------------------------------------------------------------- plain forms

def _newton_schulz(u):
    """u [count, rows, cols] in its own precision."""
    norm = u.square().sum((1, 2), keepdim=True).sqrt()
    x = u / torch.where(norm > 0, norm, torch.ones_like(norm))
    flip = x.shape[1] > x.shape[2]
    x = x.transpose(1, 2).contiguous() if flip else x
    for _ in range(NS_STEPS):
        a = torch.bmm(x, x.transpose(1, 2).contiguous())
        x = A * x + torch.bmm(B * a + C * torch.bmm(a, a), x)
    return x.transpose(1, 2).contiguous() if flip else x


def _dynamic_table():
    """Magnitudes of the 128 signed decade-tree codes."""
    t = [0.0]
    for code in range(1, 128):
        z = 7 - code.bit_length()
        p = 6 - z
        f = code - (1 << p)
        t.append((0.1 + 0.9 * ((f + 1) / 2 ** p)) * float("1e-%d" % z))
    return torch.tensor(t, dtype=torch.float64).float()


def _decode(case, codes, absmax, table):
    """Momentum values [count, numel] from codes and absmax, in absmax's precision."""
    n, numel = codes.shape
    block = case["block"]
    scale = absmax.repeat_interleave(block, 1)[:, :numel]
    if case["map"] == "linear":
        return codes.to(absmax.dtype) * (scale / torch.full_like(scale, 127.0))
    c = codes.to(torch.int64) & 0xff
    v = table.to(absmax.dtype)[c & 0x7f] * scale
    return torch.where(c >= 0x80, -v, v)


def _encode(case, m, table):
    """Codes and absmax of momentum values [count, numel]."""
    n, numel = m.shape
    block, nb = case["block"], -(-m.shape[1] // case["block"])
    absmax = torch.nn.functional.pad(m.abs(), (0, nb * block - numel)).view(n, nb, block).amax(-1)
    top = 127.0 if case["map"] == "linear" else 1.0
    inv = torch.full_like(absmax, top) / absmax
    fine = torch.isfinite(absmax) & torch.isfinite(inv)
    absmax = torch.where(fine, absmax, torch.zeros_like(absmax))
    inv = torch.where(fine, inv, torch.zeros_like(inv)).repeat_interleave(block, 1)[:, :numel]
    if case["map"] == "linear":
        return (m * inv).round().clamp(-127, 127).to(torch.int8), absmax
    table = table.to(m.dtype)
    y = m.abs() * inv
    hi = torch.searchsorted(table, y.contiguous()).clamp(1, 127)
    lo = hi - 1
    c = torch.where(table[hi] - y < y - table[lo], hi, lo)
    c = torch.where(m < 0, c | 0x80, c)
    return torch.where(c >= 0x80, c - 256, c).to(torch.int8), absmax


def _muon_group(s, i, wide):
    """One stack's step in `wide` precision: the new weights, momentum codes and absmax."""
    case = s["case"]
    g = s["grads"][i].to(wide)
    n, rows, cols = g.shape
    g = (g * s["coef"].to(wide)).view(n, -1)
    m0 = _decode(case, s["codes"][i], s["absmax"][i].to(wide), s["table"])
    # the scalars of a step are rounded to 32 bits once
    beta, rest, decay = (float(torch.tensor(v, dtype=torch.float64).float())
                         for v in (MOMENTUM, 1 - MOMENTUM, 1 - LR * WEIGHT_DECAY))
    rate = float(torch.tensor(LR * UPDATE_RMS * math.sqrt(max(rows, cols)),
                              dtype=torch.float64).float())
    cg = g * rest
    m1 = m0 * beta + cg
    u = m1 * beta + cg                  # Nesterov's look ahead
    codes, absmax = _encode(case, m1, s["table"])
    o = _newton_schulz(u.view(n, rows, cols))
    return s["w"][i].to(wide) * decay - o * rate, codes, absmax


def _muon_outputs(s, w, codes, absmax, wide=torch.float32):
    out = dict(w=w, momentum=[_decode(s["case"], c, a.to(wide), s["table"])
                              for c, a in zip(codes, absmax)])
    if s["copy"] is not None:
        out["copy"] = s["copy"]
    return out


# ---------------------------------------------------------------------- the passes

def _list(stacks):
    return [m for stack in stacks for m in stack.unbind(0)]


def _run_own(s):
    import paper_2608_11919_amd as lt
    case = s["case"]
    op = case["op"]
    if op == "orth":
        lt.lt_orthogonalize(_list(s["grads"]), _list(s["out"]), ns_steps=NS_STEPS)
        return s["out"]
    if op == "muon":
        lt.lt_muon_step(_list(s["w"]), _list(s["grads"]), _list(s["codes"]), _list(s["absmax"]),
                        case["block"], lr=LR, momentum=MOMENTUM, weight_decay=WEIGHT_DECAY,
                        ns_steps=NS_STEPS, nesterov=True, update_rms=UPDATE_RMS,
                        code_map=lt.LT_MAP_DYNAMIC if case["map"] == "dynamic"
                        else lt.LT_MAP_LINEAR, coef=s["coef"], status=s["status"],
                        params_bf16=None if s["copy"] is None else _list(s["copy"]))
        return _muon_outputs(s, s["w"], s["codes"], s["absmax"])
    n, k = case["rows"], case["cols"]
    if op == "linear":
        return lt.fp8_linear(s["x"], lt.Fp8Weight(n, k, codes=s["wq"], scales=s["ws"]))
    weight = lt.Fp8Weight.from_master(s["w"])
    y, saved = lt.fp8_linear_forward(s["x"], weight)
    dx, dw = lt.fp8_linear_backward(s["dy"], saved, weight)
    return dict(y=y, dx=dx, dw=dw)


def run(s):
    if own:
        return _run_own(s)
    case = s["case"]
    op = case["op"]
    if op == "orth":
        return [_newton_schulz(g.float()).to(torch.bfloat16) for g in s["grads"]]
    if op == "muon":
        new = [_muon_group(s, i, torch.float32) for i in range(len(s["w"]))]
        for i, (w, codes, absmax) in enumerate(new):
            s["w"][i].copy_(w)
            s["codes"][i].copy_(codes)
            s["absmax"][i].copy_(absmax)
            if s["copy"] is not None:
                s["copy"][i].copy_(w)
        return _muon_outputs(s, s["w"], s["codes"], s["absmax"])
    k, n = case["cols"], case["rows"]
    x = _values(*_rowwise(s["x"]), k)
    if op == "linear":
        return (x @ _values(s["wq"], s["ws"], k).t()).to(torch.bfloat16)
    t = case["tokens"]
    w = _values(*_square(s["w"]), k)
    y = (x @ w.t()).to(torch.bfloat16)
    dx = (_values(*_rowwise(s["dy"]), n) @ w).to(torch.bfloat16)
    dw = (_values(*_rowwise(s["dy"].t()), t) @ _values(*_rowwise(s["x"].t()), t).t())
    return dict(y=y, dx=dx, dw=dw.to(torch.bfloat16))


# ---------------------------------------------------------------------- work

def _ns_flops(r, c):
    """Products of one matrix: with n rows and m >= n columns, a step's X X^T, A A and B X,
    the first two symmetric; or all steps on n x n matrices and one product with X."""
    n, m = float(min(r, c)), float(max(r, c))
    return min(NS_STEPS * (3 * n * n * m + n ** 3), 3 * n * n * m + 4 * NS_STEPS * n ** 3)


def work(case):
    if case["op"] in ("orth", "muon"):
        groups = _groups(case)
        elems = sum(n * r * c for n, r, c in groups)
        flops = sum(n * _ns_flops(r, c) for n, r, c in groups)
        read = 2 if case["dtype"] == "bf16" else 4
        if case["op"] == "orth":
            return dict(bytes=elems * (read + 2), flops=flops)
        # gradient, weight read and written, codes read and written, the copy, absmax
        per = read + 8 + 2 + (2 if case["copy"] else 0) + 8.0 / case["block"]
        return dict(bytes=elems * per, flops=flops)
    t, k, n = case["tokens"], case["cols"], case["rows"]
    item = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "linear":
        return dict(bytes=t * k * item + n * k * (1 + 1 / GROUP) + t * n * 2, flops=2.0 * t * k * n)
    # x, dy and the master weights in; y, dx and dw out
    return dict(bytes=item * t * (k + n) + 4 * n * k + 2 * t * (k + n) + 2 * n * k,
                flops=6.0 * t * k * n)


# ---------------------------------------------------------------------- 64 bits

def _exact_orth(u):
    """The same polynomial through its products in 64 bits, matrix by matrix."""
    out = []
    for m in u.double().unbind(0):
        norm = torch.linalg.vector_norm(m)
        x = m / norm if norm > 0 else m
        for _ in range(NS_STEPS):
            g = x @ x.t() if x.shape[0] <= x.shape[1] else x.t() @ x
            p = B * g + C * (g @ g)
            x = A * x + (p @ x if x.shape[0] <= x.shape[1] else x @ p)
        out.append(x)
    return torch.stack(out)


def _exact_groups(x, square):
    """Values in 64 bits of x rounded to 3 mantissa bits under a power of two for each
    group: steps of 2^(e - 3) at magnitude 2^e, no finer than 2^-9, up to 448."""
    x = x.double()
    r, k = x.shape
    br = GROUP if square else 1
    pr, pk = -r % br, -k % GROUP
    g = torch.nn.functional.pad(x, (0, pk, 0, pr)).view((r + pr) // br, br, (k + pk) // GROUP, GROUP)
    top = g.abs().amax((1, 3), keepdim=True)
    power = torch.ceil(torch.log2(torch.where(top > 0, top, torch.full_like(top, 448.0)) / 448.0))
    # log2 may round across a whole number: put the least power right
    power = torch.where(top > 448.0 * torch.exp2(power), power + 1, power)
    power = torch.where(top <= 448.0 * torch.exp2(power - 1), power - 1, power)
    power = torch.where(top > 0, power.clamp_min(-126), torch.zeros_like(power))
    v = g * torch.exp2(-power)
    step = torch.exp2((torch.frexp(v)[1] - 4).clamp_min(-9).double())
    v = torch.round(v / step) * step * torch.exp2(power)
    return v.view(r + pr, k + pk)[:r, :k]


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "orth":
        return [_exact_orth(g) for g in s["grads"]]
    if op == "muon":
        table = _dynamic_table().double().to("cuda")
        wide = torch.float64
        w, m = [], []
        for i, g in enumerate(s["grads"]):
            n, rows, cols = g.shape
            numel, block = rows * cols, case["block"]
            code = s["codes"][i].to(torch.int64)
            scale = s["absmax"][i].to(wide).repeat_interleave(block, 1)[:, :numel]
            if case["map"] == "linear":
                m0 = code.to(wide) * scale / 127
            else:
                m0 = table[code & 0x7f] * scale * torch.where(code < 0, -1.0, 1.0).to(wide)
            cg = g.to(wide).view(n, numel) * COEF * (1 - MOMENTUM)
            m1 = MOMENTUM * m0 + cg
            o = _exact_orth((MOMENTUM * m1 + cg).view(n, rows, cols))
            w.append(s["w"][i].to(wide) * (1 - LR * WEIGHT_DECAY) -
                     LR * UPDATE_RMS * math.sqrt(max(rows, cols)) * o)
            pad = -numel % block
            top = torch.nn.functional.pad(m1.abs(), (0, pad)).view(n, -1, block).amax(-1)
            top = top.repeat_interleave(block, 1)[:, :numel]
            if case["map"] == "linear":
                m.append(torch.where(top > 0, torch.round(m1 / top * 127) * top / 127, 0.0))
            else:
                y = torch.where(top > 0, m1.abs() / top, 0.0)
                mid = (table[1:] + table[:-1]) / 2
                m.append(table[torch.searchsorted(mid, y.contiguous())] * top * torch.sign(m1))
        out = dict(w=w, momentum=m)
        if case["copy"]:
            out["copy"] = w
        return out
    x = _exact_groups(s["x"], False)
    k, n = case["cols"], case["rows"]
    if op == "linear":
        # the weight in hand is the stored one: its bytes read by their bits
        c = s["wq"].to(torch.int64)
        e, f = (c >> 3) & 15, (c & 7).double()
        v = torch.where(e > 0, (1 + f / 8) * torch.exp2((e - 7).double()), f / 8 * 2.0 ** -6)
        v = torch.where(c >= 128, -v, v)
        p = torch.exp2(s["ws"].double() - 127).repeat_interleave(GROUP, 1)[:, :v.shape[1]]
        return x @ (v * p)[:, :k].t()
    w = _exact_groups(s["w"], True)
    dy = _exact_groups(s["dy"], False)
    dw = _exact_groups(s["dy"].t(), False) @ _exact_groups(s["x"].t(), False).t()
    return dict(y=x @ w.t(), dx=dy @ w, dw=dw)
