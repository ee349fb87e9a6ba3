"""The feed-forward block's operators, as cases a measuring program can run.

Five kinds of pass, through the public entry points of ``paper_2608_11919_amd``:

* ``gated``: the gated projections of a feed-forward block in bf16, both products, the
  activation and the product of the two, as a program that answers calls them;
* ``train``: the same forward and backward, with the gradients of the tokens and of both
  weights;
* ``int8``: a linear layer's answer in 8-bit integers, a scale for each token and each
  output channel;
* ``int8_gated``: the gated projections in 8-bit integers;
* ``quantize``: a weight laid out in 8-bit integers, after a step that changed it.

Where ``own`` is false, ``run`` computes the same in elementary torch operations in 32
bits (the integer codes in 64, where a value may lie next to a border).  ``exact`` restates
the definitions in 64 bits.
"""
import math

import torch

own = False

PITCH = 128   # a row of integer codes is padded with zeros to a multiple of this
LEAST = 2.0 ** -100   # rows below this in magnitude are quantized as if they reached it


# ---------------------------------------------------------------------- cases

def listed():
    return [
        # A single token through the gated projections of the 3B-class model: the smallest call.
        dict(name="gated_one_token", op="gated", tokens=1, cols=2048, rows=11008, act="silu",
             out="bf16"),
        # A ragged prompt through a block whose sizes are no multiples of anything.
        dict(name="gated_ragged_prompt", op="gated", tokens=1237, cols=2011, rows=5003,
             act="gelu_tanh", out="f32"),
        # A few sentences of training on a small odd model.
        dict(name="train_gated_odd", op="train", tokens=301, cols=515, rows=1037, act="gelu"),
        # Eight sequences of 1024 tokens, 3B-class block, forward and backward.
        dict(name="train_gated_3b", op="train", tokens=8192, cols=2048, rows=11008, act="silu"),
        # Twice the tokens on the 27B-class block: the largest pass.
        dict(name="train_gated_27b", op="train", tokens=16384, cols=5120, rows=17408, act="silu"),
        # A single token through a feed-forward matrix of the 3B-class model, in integers.
        dict(name="int8_one_token", op="int8", tokens=1, cols=2048, rows=11008, dtype="bf16",
             out="bf16"),
        # A ragged prompt in fp32 through odd sizes.
        dict(name="int8_ragged_prompt", op="int8", tokens=1237, cols=2011, rows=5003,
             dtype="f32", out="f32"),
        # A batch of prompts through the 27B-class block's second matrix.
        dict(name="int8_prompts_27b", op="int8", tokens=8192, cols=17408, rows=5120,
             dtype="bf16", out="bf16"),
        # Sixteen sequences answering at once through the 27B-class gated projections.
        dict(name="int8_gated_16_tokens", op="int8_gated", tokens=16, cols=5120, rows=17408,
             dtype="bf16", act="silu", out="bf16"),
        # A prompt of 4096 tokens through the 3B-class gated projections.
        dict(name="int8_gated_prompt", op="int8_gated", tokens=4096, cols=2048, rows=11008,
             dtype="bf16", act="silu", out="bf16"),
        # A small odd matrix and the fp32 master weights of a 27B-class one, laid out for
        # answering after a step.
        dict(name="int8_weight_odd", op="quantize", cols=515, rows=1037, dtype="bf16"),
        dict(name="int8_weight_27b", op="quantize", cols=5120, rows=17408, dtype="f32"),
    ]


ACTIVATIONS = ["silu", "gelu", "gelu_tanh", "relu"]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed kinds, over their whole ranges."""
    op = rng.choice(["gated", "gated", "train", "train", "int8", "int8", "int8_gated",
                     "int8_gated", "quantize"])
    c = dict(op=op, cols=_log_int(rng, 64, 5120), rows=_log_int(rng, 64, 17408))
    if op in ("int8", "quantize") and rng.random() < 0.5:
        c["cols"], c["rows"] = c["rows"], c["cols"]
    if rng.random() < 0.6:      # model dimensions are mostly multiples of 64
        c["cols"], c["rows"] = -(-c["cols"] // 64) * 64, -(-c["rows"] // 64) * 64
    if op in ("int8", "int8_gated", "quantize"):
        c["dtype"] = rng.choice(["bf16", "bf16", "f32"])
    if op != "quantize":
        c["tokens"] = _log_int(rng, 64, 12288) if op == "train" else _log_int(rng, 1, 8192)
        if op != "train":
            c["out"] = rng.choice(["bf16", "bf16", "f32"])
        if op != "int8":
            c["act"] = rng.choice(["silu"] + ACTIVATIONS)
    return c


# ---------------------------------------------------------------------- inputs

_DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


def _codes(x):
    """x [R, K] as 8-bit integers under a scale for each row: codes [R, K] in x's order, as
    whole numbers in 32-bit floats, and scales [R].  The code is x times fp32(127 / most)
    rounded to the nearest integer, ties to even; the scale is fp32(most / 127)."""
    most = x.float().abs().amax(1).clamp_min(LEAST)
    top = torch.full_like(most, 127.0)  # quotients of tensors are rounded once
    codes = (x.double() * (top / most).double().unsqueeze(1)).round().float()
    return codes, most / top


def _weight(w):
    """The stored form of a weight: bytes padded to a multiple of 128 columns, scales."""
    codes, scales = _codes(w)
    pad = -w.shape[1] % PITCH
    return torch.nn.functional.pad(codes.to(torch.int8), (0, pad)).contiguous(), scales


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)

    def randn(rows, cols):
        return torch.randn(rows, cols, device="cuda", generator=gen)

    op, k, n = case["op"], case["cols"], case["rows"]
    s = dict(case=case)
    if op == "quantize":
        s["w"] = (randn(n, k) / math.sqrt(k)).to(_DTYPE[case["dtype"]])
        return s
    t = case["tokens"]
    # activations after a norm: near one, with a few channels far above the rest
    loud = torch.rand(k, device="cuda", generator=gen) < 0.01
    x = randn(t, k) * torch.where(loud, 8.0, 1.0)
    s["x"] = x.to(_DTYPE[case.get("dtype", "bf16")])
    names = ["w"] if op == "int8" else ["gate", "up"]
    for name in names:
        w = randn(n, k) / math.sqrt(k)
        # a program that answers keeps the integer weights, one that trains the bf16 ones
        s[name] = _weight(w) if op.startswith("int8") else w.to(torch.bfloat16)
    if op == "train":
        s["dh"] = (randn(t, n) * 1e-3).to(torch.bfloat16)
    return s


# ---------------------------------------------------------------------- plain forms

def _act(name, g):
    if name == "silu":
        return g / (1 + torch.exp(-g))
    if name == "gelu":
        return g * 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return g * 0.5 * (1 + torch.tanh(math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)))
    return g.clamp_min(0)


def _slope(name, g):
    """The activation's derivative."""
    if name == "silu":
        p = 1 / (1 + torch.exp(-g))
        return p * (1 + g * (1 - p))
    if name == "gelu":
        return (0.5 * (1 + torch.erf(g * math.sqrt(0.5))) +
                g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi))
    if name == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        h = torch.tanh(c * (g + 0.044715 * g ** 3))
        return 0.5 * (1 + h) + 0.5 * g * (1 - h * h) * c * (1 + 3 * 0.044715 * g * g)
    return (g > 0).to(g.dtype)


def _run_own(s):
    import paper_2608_11919_amd as lt
    case = s["case"]
    op, k, n = case["op"], case["cols"], case["rows"]
    if op == "quantize":
        w = lt.Int8Weight.from_master(s["w"])
        return dict(values=w.codes[:, :k] * w.scales.unsqueeze(1), scales=w.scales)
    if op == "train":
        h, saved = lt.gated_linear_forward(s["x"], s["gate"], s["up"], case["act"])
        dx, dgate, dup = lt.gated_linear_backward(s["dh"], saved, s["x"], s["gate"], s["up"])
        return dict(h=h, dx=dx, dgate=dgate, dup=dup)
    out = _DTYPE[case["out"]]
    if op == "gated":
        return lt.gated_linear(s["x"], s["gate"], s["up"], case["act"], out_dtype=out)
    if op == "int8":
        return lt.int8_linear(s["x"], lt.Int8Weight(n, k, *s["w"]), out_dtype=out)
    return lt.int8_gated_linear(s["x"], lt.Int8Weight(n, k, *s["gate"]),
                                lt.Int8Weight(n, k, *s["up"]), case["act"], out_dtype=out)


def run(s):
    if own:
        return _run_own(s)
    case = s["case"]
    op, k = case["op"], case["cols"]
    if op == "quantize":
        codes, scales = _codes(s["w"])
        return dict(values=codes * scales.unsqueeze(1), scales=scales)
    if op in ("int8", "int8_gated"):
        x, sx = _codes(s["x"])

        def product(w):
            return (x @ w[0][:, :k].float().t()) * sx.unsqueeze(1) * w[1]

        if op == "int8":
            return product(s["w"]).to(_DTYPE[case["out"]])
        return (_act(case["act"], product(s["gate"])) * product(s["up"])).to(_DTYPE[case["out"]])
    x, gate, up = s["x"].float(), s["gate"].float(), s["up"].float()
    g, u = x @ gate.t(), x @ up.t()
    a = _act(case["act"], g)
    if op == "gated":
        return (a * u).to(_DTYPE[case["out"]])
    dh = s["dh"].float()
    h = (a * u).to(torch.bfloat16)
    dg, du = dh * u * _slope(case["act"], g), dh * a
    return dict(h=h, dx=(dg @ gate + du @ up).to(torch.bfloat16),
                dgate=(dg.t() @ x).to(torch.bfloat16), dup=(du.t() @ x).to(torch.bfloat16))


# ---------------------------------------------------------------------- work

def work(case):
    op, k, n = case["op"], case["cols"], case["rows"]
    item = 4 if case.get("dtype") == "f32" else 2
    if op == "quantize":
        # the weight in; the values that the codes stand for and the scales out
        return dict(bytes=item * n * k + n * k + 4 * n, flops=0.0)
    t = case["tokens"]
    out = 4 if case.get("out") == "f32" else 2
    if op == "train":
        # x, dh and both weights in; h, dx and both gradients out
        return dict(bytes=2 * (2 * t * k + 2 * t * n + 4 * n * k), flops=12.0 * t * k * n)
    weights = 1 if op == "int8" else 2
    each = 2 if op == "gated" else 1
    scales = 4 * n * weights if op != "gated" else 0
    return dict(bytes=item * t * k + weights * each * n * k + scales + out * t * n,
                flops=2.0 * weights * t * k * n)


# ---------------------------------------------------------------------- 64 bits

def _exact_act(name, g):
    """The activation and its derivative."""
    if name == "relu":
        return torch.where(g > 0, g, 0.0), torch.where(g > 0, 1.0, 0.0).double()
    if name == "gelu":
        cdf = torch.special.ndtr(g)
        return g * cdf, cdf + g * torch.exp(-g * g / 2) * (2 * math.pi) ** -0.5
    # both others are g times a logistic function of an odd polynomial p
    c, d = (2 * (2 / math.pi) ** 0.5, 2 * 0.044715 * (2 / math.pi) ** 0.5) \
        if name == "gelu_tanh" else (1.0, 0.0)
    s = torch.sigmoid(g * (c + d * g * g))
    return g * s, s + g * s * (1 - s) * (c + 3 * d * g * g)


def _exact_codes(x):
    """Codes and scales by their definition: its two quotients are rounded to 32 bits, the
    product of value and quotient is exact in 64."""
    x = x.double()
    most = torch.maximum(x.amax(1), -x.amin(1))
    most = torch.where(most < LEAST, LEAST, most)
    factor, scale = (127 / most).float().double(), (most / 127).float().double()
    v = x * factor[:, None]
    low = torch.floor(v)
    rest = v - low
    up = (rest > 0.5) | ((rest == 0.5) & (low.remainder(2) == 1))
    return low + up.double(), scale


def exact(case, seed):
    s = prepare(case, seed)
    op, k = case["op"], case["cols"]
    if op == "quantize":
        codes, scales = _exact_codes(s["w"])
        return dict(values=codes * scales[:, None], scales=scales)
    if op in ("int8", "int8_gated"):
        codes, scales = _exact_codes(s["x"])
        x = codes * scales[:, None]
        y = [x @ (s[w][0][:, :k].double() * s[w][1].double()[:, None]).t()
             for w in (["w"] if op == "int8" else ["gate", "up"])]
        return y[0] if op == "int8" else _exact_act(case["act"], y[0])[0] * y[1]
    x, gate, up = s["x"].double(), s["gate"].double(), s["up"].double()
    g, u = x @ gate.t(), x @ up.t()
    a, slope = _exact_act(case["act"], g)
    if op == "gated":
        return a * u
    h = a * u
    dh = s["dh"].double()
    dg = u.mul_(slope).mul_(dh)
    du = a.mul_(dh)
    return dict(h=h, dx=dg @ gate + du @ up, dgate=dg.t() @ x, dup=du.t() @ x)
