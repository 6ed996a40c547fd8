"""Operator cases: decoder linears in microscaled formats, what forms their inputs, and the choice of the next word.

A microscaled matrix (MX) has blocks of 32 consecutive elements of a row, each block with a scale that is a power of two (one
byte, E8M0) and elements of 4 bits (E2M1) or 8 bits (E4M3).  The scale is the smallest power of two, at least 2^-127, that leaves
no element of the block above the element type's largest value (6 and 448); elements are rounded to nearest, ties to even.

  norm      one `add_rmsnorm` call: the residual stream and a layer's output are added and the sum normalised, into a linear's
            input in its own type or in MX 8-bit values.
  quantize  one `mx_quantize` call: 16- or 32-bit activations to MX 8-bit values, with or without the gated product of the gate
            and up projections.
  convert   one `mx_quantize` and one `mx_dequantize` call: a weight matrix to MX values and back, as a converter does that
            looks at what a format makes of a checkpoint.
  linear    one `mx_linear` call: y = x W^T with MX 4-bit weights and MX 8- or 4-bit activations.
  project   one `mx_quantize` and one `mx_linear` call: the same from activations in 16 bits.
  sample    one `sample_logits` call: the next word from given random numbers, with temperature, top-k, top-p and min-p.

Sizes are those of the 8B-class decoder that the tests and the benchmark use, and generic ones.  `draw` spreads sizes, ragged
ones among them, over the same ranges.
"""

from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-5


def listed():
    return [
        # One token's residual addition and norm ahead of the QKV projection: latency is all there is.
        dict(name="norm_1", kind="norm", rows=1, dim=4096, residual=True, out=8, dtype="f16"),
        # A small batch of a model with an odd width, without a residual (the first layer), into the 16-bit linears.
        dict(name="norm_77", kind="norm", rows=77, dim=2080, residual=False, out=16, dtype="bf16"),
        # A prompt of 8192 tokens.
        dict(name="norm_8192", kind="norm", rows=8192, dim=4096, residual=True, out=8, dtype="bf16"),
        # The down projection's input of a 2048-token prompt, from the gate and up projections' output.
        dict(name="quantize_gated_2048", kind="quantize", rows=2048, cols=14336, gated=True, dtype="f16"),
        # A checkpoint's down projection to 4 bits and back.
        dict(name="convert_4096", kind="convert", rows=4096, cols=14336, bits=4, dtype="bf16"),
        # One token through the gate and up projections: the weights' bytes.
        dict(name="linear_1", kind="linear", n=28672, k=4096, m=1, bits=8, dtype="f16"),
        # A server's decoding step of 33 sequences through the down projection.
        dict(name="linear_33", kind="linear", n=4096, k=14336, m=33, bits=8, dtype="bf16"),
        # Ragged in every size: a slice of a projection, a chunk of 777 tokens, 4-bit activations.
        dict(name="linear_777", kind="linear", n=1003, k=2080, m=777, bits=4, dtype="f16"),
        # The largest: a prompt of 8192 tokens through the gate and up projections.
        dict(name="linear_8192", kind="linear", n=28672, k=4096, m=8192, bits=8, dtype="f16"),
        # A prompt of 4096 tokens through the down projection, its input rounded to 4 bits on the way.
        dict(name="project_4096", kind="project", n=4096, k=14336, m=4096, bits=4, dtype="bf16"),
        # One sequence's next word from a 128256-word vocabulary, the usual settings of a chat.
        dict(name="sample_1", kind="sample", rows=1, vocab=128256, settings="k50p95", masked=0.0, dtype="f16"),
        # A large batch in 32 bits, every row with settings of its own, some words not allowed.
        dict(name="sample_256", kind="sample", rows=256, vocab=100277, settings="mixed", masked=0.3, dtype="f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    kind = rng.choice(["norm"] * 3 + ["quantize"] * 2 + ["convert"] + ["linear"] * 5 + ["project"] * 2 + ["sample"] * 4)
    dtype = rng.choice(["f16", "f16", "bf16", "bf16", "f32"])
    while True:
        if kind == "norm":
            case = dict(kind=kind, rows=_log_int(rng, 1, 8192), dim=32 * _log_int(rng, 1, 512), residual=rng.random() < 0.7, out=rng.choice([8, 8, 16]),
                        dtype=dtype)
        elif kind == "quantize":
            case = dict(kind=kind, rows=_log_int(rng, 1, 8192), cols=32 * _log_int(rng, 1, 512), gated=rng.random() < 0.5, dtype=dtype)
        elif kind == "convert":
            case = dict(kind=kind, rows=_log_int(rng, 1, 28672), cols=32 * _log_int(rng, 1, 512), bits=rng.choice([4, 4, 8]), dtype=dtype)
        elif kind in ("linear", "project"):
            case = dict(kind=kind, n=_log_int(rng, 16, 32768), k=32 * _log_int(rng, 1, 512), m=rng.choice([1, rng.randint(2, 64), _log_int(rng, 1, 8192)]),
                        bits=rng.choice([8, 4]), dtype=rng.choice(["f16", "bf16"]))
        else:
            case = dict(kind=kind, rows=_log_int(rng, 1, 256), vocab=_log_int(rng, 500, 200000), settings=rng.choice(["k50p95", "mixed", "top_p", "min_p", "all"]),
                        masked=rng.choice([0.0, round(rng.uniform(0.0, 0.9), 2)]), dtype=dtype)
        w = work(case)
        if w["bytes"] <= 1 << 29 and w["flops"] <= work(listed()[8])["flops"]:
            return case


# ------------------------------------------------------------------ inputs


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _activations(g, rows, cols):
    """A residual stream's values: a few columns are much larger than the others."""
    large = torch.rand(cols, generator=g, device="cuda") < 0.004
    return _normal(g, rows, cols).mul_(torch.where(large, 20.0, 1.0))


def _weights(g, n, k):
    return _normal(g, n, k).mul_(torch.rand((n, 1), generator=g, device="cuda").add_(0.5)).mul_(1.0 / math.sqrt(k))


def _empty(rows, cols, bits):
    """Room for an MX matrix; rows of scales are padded to 16 bytes."""
    codes = torch.empty((rows, cols // 2), dtype=torch.uint8, device="cuda") if bits == 4 else torch.empty((rows, cols), dtype=torch.float8_e4m3fn, device="cuda")
    return codes, torch.zeros((rows, -(-cols // 512) * 16), dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)


def prepare(case, seed):
    g, kind, dtype = _generator(seed), case["kind"], DTYPES[case["dtype"]]
    d = dict(case)
    if kind == "norm":
        rows, dim = case["rows"], case["dim"]
        d.update(x=_activations(g, rows, dim).to(dtype), weight=_normal(g, dim).mul_(0.1).add_(1.0).to(dtype),
                 residual=_activations(g, rows, dim).mul_(3.0).to(dtype) if case["residual"] else None,
                 total=torch.empty((rows, dim), dtype=dtype, device="cuda") if case["residual"] else None)
        if case["out"] == 16:
            d.update(y=torch.empty((rows, dim), dtype=dtype, device="cuda"), codes=None, scales=None)
        else:
            d.update(y=None, **dict(zip(("codes", "scales"), _empty(rows, dim, 8))))
    elif kind == "quantize":
        d.update(x=_activations(g, case["rows"], case["cols"] * (2 if case["gated"] else 1)).to(dtype),
                 **dict(zip(("codes", "scales"), _empty(case["rows"], case["cols"], 8))))
    elif kind == "convert":
        d.update(x=_weights(g, case["rows"], case["cols"]).to(dtype), y=torch.empty((case["rows"], case["cols"]), dtype=dtype, device="cuda"),
                 **dict(zip(("codes", "scales"), _empty(case["rows"], case["cols"], case["bits"]))))
    elif kind in ("linear", "project"):
        n, k, m, bits = case["n"], case["k"], case["m"], case["bits"]
        d["w_codes"], d["w_scales"] = _empty(n, k, 4)
        _store(_quantized(_weights(g, n, k), 4), d["w_codes"], d["w_scales"])
        x = _activations(g, m, k)
        d["x_codes"], d["x_scales"] = _empty(m, k, bits)
        if kind == "linear":
            _store(_quantized(x, bits), d["x_codes"], d["x_scales"])
        else:
            d["x"] = x.to(dtype)
        d["y"] = torch.empty((m, n), dtype=dtype, device="cuda")
        if own:
            from paper_2412_15803_amd import wq

            d["workspace"] = wq.mx_linear_workspace(d["w_codes"], d["x_codes"])
    else:
        rows, vocab, settings = case["rows"], case["vocab"], case["settings"]
        logits = _normal(g, rows, vocab).mul_(3.0)
        logits[torch.rand((rows, vocab), generator=g, device="cuda") < case["masked"]] = -math.inf
        d.update(logits=logits.to(dtype), random=torch.rand(rows, generator=g, device="cuda"), token=torch.empty(rows, dtype=torch.int32, device="cuda"),
                 share=torch.empty(rows, device="cuda"), temperature=torch.full((rows,), 0.8, device="cuda"), top_k=None, top_p=None, min_p=None)
        pick = lambda chance: torch.rand(rows, generator=g, device="cuda") < chance  # noqa: E731
        unit = lambda lo, hi: torch.rand(rows, generator=g, device="cuda").mul_(hi - lo).add_(lo)  # noqa: E731
        if settings == "k50p95":
            d.update(top_k=torch.full((rows,), 50, dtype=torch.int32, device="cuda"), top_p=torch.full((rows,), 0.95, device="cuda"))
        elif settings == "top_p":
            d["top_p"] = unit(0.8, 0.98)
        elif settings == "min_p":
            d["min_p"] = unit(0.02, 0.1)
        elif settings == "mixed":
            d.update(temperature=torch.where(pick(0.1), 0.0, unit(0.5, 1.3)), top_p=torch.where(pick(0.5), 1.0, unit(0.8, 0.98)),
                     top_k=torch.where(pick(0.5), 0, unit(0.0, 7.0).exp_()).to(torch.int32), min_p=torch.where(pick(0.7), 0.0, unit(0.02, 0.1)))
        if own:
            from paper_2412_15803_amd import wq

            d["workspace"] = wq.sample_workspace(d["logits"])
    return d


# --------------------------------------------------------------------- run


def run(d):
    return (_run_own if own else _PLAIN[d["kind"]])(d)


def _mx_values(d):
    """The MX values as they lie, elements and scales."""
    return dict(codes=d["codes"], scales=d["scales"][:, :d["codes"].shape[1] // 32])


def _run_own(d):
    from paper_2412_15803_amd import wq

    kind = d["kind"]
    if kind == "norm":
        wq.add_rmsnorm(d["x"], d["weight"], EPS, out=d["y"], residual=d["residual"], total=d["total"], codes=d["codes"], scales=d["scales"])
        out = dict(total=d["total"]) if d["total"] is not None else {}
        return dict(out, y=d["y"]) if d["out"] == 16 else dict(out, **_mx_values(d))
    if kind == "quantize":
        wq.mx_quantize(d["x"], d["codes"], d["scales"], gated=d["gated"])
        return _mx_values(d)
    if kind == "convert":
        wq.mx_quantize(d["x"], d["codes"], d["scales"])
        wq.mx_dequantize(d["codes"], d["scales"], d["y"])
        return d["y"]
    if kind in ("linear", "project"):
        if kind == "project":
            wq.mx_quantize(d["x"], d["x_codes"], d["x_scales"])
        wq.mx_linear(d["w_codes"], d["w_scales"], d["x_codes"], d["x_scales"], d["y"], workspace=d["workspace"])
        return d["y"]
    wq.sample_logits(d["logits"], d["random"], d["token"], temperature=d["temperature"], top_k=d["top_k"], top_p=d["top_p"], min_p=d["min_p"], share=d["share"],
                     workspace=d["workspace"])
    return dict(token=d["token"], share=d["share"])


# ------------------------------------------------------------- plain forms


def _quantized(v, bits):
    """Elements [rows, cols / 32, 32] over their scales, rounded to the element type but still fp32, and the scales' exponents."""
    v = v.float().view(v.shape[0], -1, 32)
    fraction, exponent = torch.frexp(v.abs().amax(-1))  # largest = fraction 2^exponent, 1/2 <= fraction < 1
    if bits == 4:
        exponent = exponent - 3 + (fraction > 0.75).to(exponent.dtype)  # 6 = 0.75 * 2^3
    else:
        exponent = exponent - 9 + (fraction > 0.875).to(exponent.dtype)  # 448 = 0.875 * 2^9
    exponent = torch.where(fraction == 0, -127, exponent).clamp(min=-127)
    v = torch.ldexp(v, -exponent[..., None])
    if bits == 8:
        return v.to(torch.float8_e4m3fn).float(), exponent
    # Steps of 1/2 below 2, of 1 from there to 4, and of 2 above.
    size = v.abs()
    step = torch.where(size < 2, 0.5, torch.where(size < 4, 1.0, 2.0))
    return torch.round(v / step) * step, exponent


def _store(quantized, codes, scales):
    """Writes _quantized's values as an MX matrix."""
    v, exponent = quantized
    if codes.dtype == torch.uint8:
        size = v.abs().view(v.shape[0], -1)
        code = torch.where(size < 2, size * 2, torch.where(size < 4, size + 2, size / 2 + 4)).to(torch.uint8)
        code |= torch.signbit(v).view(v.shape[0], -1).to(torch.uint8) << 3
        codes.copy_(code[:, 0::2] | code[:, 1::2] << 4)
    else:
        codes.copy_(v.view(v.shape[0], -1).to(torch.float8_e4m3fn))
    scales.view(torch.uint8)[:, :exponent.shape[1]] = (exponent + 127).to(torch.uint8)


def _values(codes, scales):
    """What an MX matrix stands for, in 32 bits."""
    if codes.dtype == torch.uint8:
        one = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device="cuda")
        one = torch.cat([one, -one])
        pair = torch.stack([one.repeat(16), one.repeat_interleave(16)], -1)
        v = pair[codes.int()].view(codes.shape[0], -1, 32)
    else:
        v = codes.float().view(codes.shape[0], -1, 32)
    exponent = scales.view(torch.uint8)[:, :v.shape[1]].int() - 127
    return torch.ldexp(v, exponent[..., None]).view(codes.shape[0], -1)


def _plain_norm(d):
    s = d["x"].float()
    if d["residual"] is not None:
        s = s + d["residual"].float()
    y = s / torch.sqrt(s.square().mean(-1, keepdim=True) + EPS) * d["weight"].float()
    out = dict(total=s.to(d["x"].dtype)) if d["residual"] is not None else {}
    if d["out"] == 16:
        return dict(out, y=y.to(d["x"].dtype))
    _store(_quantized(y, 8), d["codes"], d["scales"])
    return dict(out, **_mx_values(d))


def _plain_quantize(d):
    x = d["x"].float()
    if d["gated"]:
        gate, up = x[:, :d["cols"]], x[:, d["cols"]:]
        x = gate / (1 + torch.exp(-gate)) * up
    _store(_quantized(x, 8), d["codes"], d["scales"])
    return _mx_values(d)


def _plain_convert(d):
    v, exponent = _quantized(d["x"], d["bits"])
    return torch.ldexp(v, exponent[..., None]).view(d["x"].shape).to(d["x"].dtype)


def _plain_linear(d):
    return torch.matmul(_values(d["x_codes"], d["x_scales"]), _values(d["w_codes"], d["w_scales"]).t()).to(d["y"].dtype)


def _plain_project(d):
    v, exponent = _quantized(d["x"], d["bits"])
    return torch.matmul(torch.ldexp(v, exponent[..., None]).view(d["x"].shape), _values(d["w_codes"], d["w_scales"]).t()).to(d["y"].dtype)


def _plain_sample(d):
    """In 64 bits: the random number may lie next to a border between two words, a sum next to top_p."""
    x = d["logits"].double()
    rows, vocab = x.shape
    greedy = d["temperature"] == 0
    t = torch.where(greedy, 1.0, d["temperature"].double())[:, None]
    x, order = x.sort(dim=-1, descending=True, stable=True)  # of equal words the lowest comes first
    w = torch.exp((x - x[:, :1]) / t)
    rank = torch.arange(vocab, device="cuda")
    keep = rank < torch.where(greedy, 1, vocab)[:, None]
    if d["top_k"] is not None:
        keep &= (rank < d["top_k"][:, None]) | (d["top_k"] <= 0)[:, None]
    w = w * keep
    total = w.cumsum(-1)
    if d["top_p"] is not None:
        before = torch.cat([torch.zeros((rows, 1), dtype=torch.float64, device="cuda"), total[:, :-1]], -1)
        w = w * ((before < d["top_p"].double()[:, None] * total[:, -1:]) | (d["top_p"] >= 1)[:, None])
    if d["min_p"] is not None:
        w = w * (w >= d["min_p"].double()[:, None])
    w = torch.zeros_like(w).scatter_(1, order, w)
    total = w.cumsum(-1)
    token = (total <= d["random"].double()[:, None] * total[:, -1:]).sum(-1, keepdim=True)
    return dict(token=token.squeeze(1).to(torch.int32), share=(w.gather(1, token) / total[:, -1:]).squeeze(1).float())


_PLAIN = dict(norm=_plain_norm, quantize=_plain_quantize, convert=_plain_convert, linear=_plain_linear, project=_plain_project, sample=_plain_sample)


# -------------------------------------------------------------------- work


def _mx_bytes(rows, cols, bits):
    return rows * (cols * bits // 8 + cols // 32)


def work(case):
    kind, size = case["kind"], DTYPES[case["dtype"]].itemsize
    if kind == "norm":
        rows, dim = case["rows"], case["dim"]
        y = rows * dim * size if case["out"] == 16 else _mx_bytes(rows, dim, 8)
        return dict(bytes=rows * dim * size * (3 if case["residual"] else 1) + dim * size + y, flops=6 * rows * dim)
    if kind == "quantize":
        rows, cols = case["rows"], case["cols"]
        return dict(bytes=rows * cols * size * (2 if case["gated"] else 1) + _mx_bytes(rows, cols, 8), flops=2 * rows * cols)
    if kind == "convert":
        rows, cols = case["rows"], case["cols"]
        return dict(bytes=2 * rows * cols * size + _mx_bytes(rows, cols, case["bits"]), flops=3 * rows * cols)
    if kind in ("linear", "project"):
        n, k, m = case["n"], case["k"], case["m"]
        x = m * k * size if kind == "project" else _mx_bytes(m, k, case["bits"])
        return dict(bytes=_mx_bytes(n, k, 4) + x + m * n * size, flops=2 * m * n * k)
    return dict(bytes=case["rows"] * (case["vocab"] * size + 28), flops=4 * case["rows"] * case["vocab"])


# ----------------------------------------------------------------- 64 bits


def exact(case, seed):
    d = prepare(case, seed)
    kind = case["kind"]
    if kind == "norm":
        s = d["x"].double() + (d["residual"].double() if case["residual"] else 0)
        y = s * (torch.linalg.vector_norm(s, dim=-1, keepdim=True).square() / case["dim"] + EPS).pow(-0.5) * d["weight"].double()
        out = dict(total=s) if case["residual"] else {}
        return dict(out, y=y) if case["out"] == 16 else dict(out, **_exact_codes(y))
    if kind == "quantize":
        x = d["x"].double()
        return _exact_codes(torch.sigmoid(x[:, :case["cols"]]) * x[:, :case["cols"]] * x[:, case["cols"]:] if case["gated"] else x)
    if kind == "convert":
        return _exact_rounded(d["x"].double(), case["bits"])
    if kind in ("linear", "project"):
        x = _exact_values(d["x_codes"], d["x_scales"]) if kind == "linear" else _exact_rounded(d["x"].double(), case["bits"])
        w = _exact_values(d["w_codes"], d["w_scales"])
        y = torch.empty((case["m"], case["n"]), dtype=torch.float64, device="cuda")
        for at in range(0, case["n"], 4096):  # a slice of the weights at a time
            y[:, at:at + 4096] = x @ w[at:at + 4096].t().contiguous()
        return y
    return _exact_sample(d)


def _exact_scale(blocks, top):
    """The smallest power of two from 2^-127 on that brings every element of a block to `top` or below."""
    x = torch.exp2(torch.ceil(torch.log2(blocks.abs().amax(-1, keepdim=True) / top)).clamp(-127, 127))
    x = torch.where(blocks.abs().amax(-1, keepdim=True) > top * x, 2 * x, x)  # should the logarithm have been rounded
    return torch.where((blocks.abs().amax(-1, keepdim=True) <= top * x / 2) & (x > 2.0 ** -127), x / 2, x)


def _exact_codes(y):
    """The elements before their rounding to 8 bits.  The scales are whole powers of two, which have no more exact value."""
    blocks = y.view(y.shape[0], -1, 32)
    return dict(codes=(blocks / _exact_scale(blocks, 448.0)).view(y.shape), scales=None)


def _exact_rounded(y, bits):
    """The nearest representable values, found among all of the type's."""
    top = 6.0 if bits == 4 else 448.0
    if bits == 4:
        grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device="cuda")
    else:
        grid = torch.arange(127, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn).double()
    middle = (grid[1:] + grid[:-1]) / 2
    out = torch.empty_like(y)
    for at in range(0, y.shape[0], 1024):
        blocks = y[at:at + 1024].view(-1, y.shape[1] // 32, 32)
        scale = _exact_scale(blocks, top)
        size = (blocks / scale).abs()
        below, above = torch.searchsorted(middle, size, right=False), torch.searchsorted(middle, size, right=True)
        # At a middle the two differ: the even one holds.
        near = torch.where(below % 2 == 0, below, above)
        out[at:at + 1024] = (grid[near] * torch.sign(blocks) * scale).view(-1, y.shape[1])
    return out


def _exact_values(codes, scales):
    rows = codes.shape[0]
    if codes.dtype == torch.uint8:
        v = torch.stack([codes & 15, codes >> 4], -1).view(rows, -1)
        e, m = (v >> 1 & 3).double(), (v & 1).double()
        v = torch.where(e == 0, m / 2, (1 + m / 2) * torch.exp2(e - 1)) * (1 - 2 * (v >> 3).double())
    else:
        v = codes.double()
    return (v.view(rows, -1, 32) * torch.exp2(scales.view(torch.uint8)[:, :v.shape[1] // 32, None].double() - 127)).view(rows, -1)


def _exact_sample(d):
    """Row by row, the words that stay picked by their ranks."""
    tokens, shares = [], []
    for i, x in enumerate(d["logits"].double()):
        t = float(d["temperature"][i])
        if t == 0:
            tokens.append(int(torch.nonzero(x == x.max())[0]))
            shares.append(1.0)
            continue
        value, word = torch.sort(x / t, descending=True, stable=True)
        p = torch.softmax(value, -1)
        if d["top_k"] is not None and 0 < int(d["top_k"][i]) < len(x):
            p[int(d["top_k"][i]):] = 0
            p = p / p.sum()
        most = p[0].clone()
        if d["top_p"] is not None and float(d["top_p"][i]) < 1:
            p[int((p.cumsum(-1) - p < float(d["top_p"][i])).sum()):] = 0
        if d["min_p"] is not None:
            p[p < float(d["min_p"][i]) * most] = 0
        q = torch.zeros_like(p)
        q[word] = p / p.sum()
        token = int(torch.searchsorted(q.cumsum(-1), d["random"][i].double(), right=True))
        tokens.append(token)
        shares.append(float(q[token]))
    return dict(token=torch.tensor(tokens, dtype=torch.int32, device="cuda"), share=torch.tensor(shares, dtype=torch.float64, device="cuda"))
