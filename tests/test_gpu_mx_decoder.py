"""The microscaled operators, the norm and the choice of words together, as the decoding example runs them.

Every call of the run is checked by itself: what it wrote against its formula in
float64 on what it was given, so that a call that reads its inputs too early, or
another's workspace, is found wherever it is in the run.  The bounds are those of the operators:
rounding to a step of the results' type (half of it relative to a value), the sums' fp32 roundings, and, where
a value lies that close to a border between two elements of a format, the other of the two."""

from __future__ import annotations

import math

import numpy as np
import pytest
import torch

import mx_model as mm
from gpu_util import announce, require_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    require_gpu()


def values(codes, scales):
    bits = 4 if codes.dtype is torch.uint8 else 8
    c = codes.view(torch.uint8).cpu().numpy()
    c = mm.unpack(c) if bits == 4 else c
    return torch.from_numpy(mm.values(c, scales.view(torch.uint8).cpu().numpy()[:, :c.shape[1] // 32], bits)), bits


def check_rounded(v, codes, scales, slack):
    """codes and scales against v (float64), known to a relative `slack`: each element within half a step of its
    block's scale, which may be the next one up or down where the largest element is that close to its border."""
    got, bits = values(codes, scales)
    top, smallest = (6.0, 0.5) if bits == 4 else (448.0, 2.0 ** -9)
    most = v.view(v.shape[0], -1, 32).abs().amax(-1)
    byte = scales.view(torch.uint8).cpu()[:, :most.shape[1]].double()
    scale = torch.exp2(byte - 127)
    assert bool((most * (1 - slack) <= top * scale).all()) and bool(((most * (1 + slack) > top * scale / 2) | (byte == 0)).all())
    wide = scale.repeat_interleave(32, 1)
    step = torch.clamp(torch.exp2(torch.floor(torch.log2(got.abs().clamp_min(1e-300) / wide)) - (1 if bits == 4 else 3)), min=smallest) * wide
    assert bool(((got - v).abs() <= step / 2 + slack * v.abs()).all())


class Checked:
    """wq with every call of the operators compared."""

    def __init__(self, wq):
        self.wq, self.calls = wq, {}

    def __getattr__(self, name):
        return getattr(self.wq, name)

    def count(self, name):
        self.calls[name] = self.calls.get(name, 0) + 1

    def add_rmsnorm(self, x, weight, eps, out=None, residual=None, total=None, codes=None, scales=None):
        s = x.double().cpu() + (0 if residual is None else residual.double().cpu())
        self.wq.add_rmsnorm(x, weight, eps, out=out, residual=residual, total=total, codes=codes, scales=scales)
        v = s / torch.sqrt(s.square().mean(-1, keepdim=True) + eps) * weight.double().cpu()
        if total is not None:
            assert torch.equal(total.cpu(), s.float().to(total.dtype))  # (Sums of two fp16 numbers are fp32 numbers.)
        check_rounded(v, codes, scales, 2.0 ** -18)
        self.count("norm")

    def mx_quantize(self, x, codes, scales, gated=False):
        v = x.double().cpu()
        if gated:
            gate, up = v.chunk(2, -1)
            v = gate / (1 + torch.exp(-gate)) * up
        self.wq.mx_quantize(x, codes, scales, gated=gated)
        check_rounded(v, codes, scales, 2.0 ** -19 if gated else 0.0)
        self.count("gated" if gated else "quantize")

    def mx_linear(self, w_codes, w_scales, x_codes, x_scales, y):
        self.wq.mx_linear(w_codes, w_scales, x_codes, x_scales, y)
        w, x = values(w_codes, w_scales)[0], values(x_codes, x_scales)[0]
        want, weight = x @ w.t(), x.abs() @ w.abs().t()
        assert bool(((y.double().cpu() - want).abs() <= 2.0 ** -11 * want.abs() + 2.0 ** -13 * weight + 2.0 ** -25).all())
        self.count("linear")

    def sample_logits(self, logits, random, token, temperature=None, top_k=None, top_p=None, min_p=None, share=None, workspace=None):
        import sample_model as sm

        self.wq.sample_logits(logits, random, token, temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p, share=share, workspace=workspace)
        for i, row in enumerate(logits.double().cpu().numpy()):
            of = lambda t, default: default if t is None else t[i].item()  # noqa: E731
            weights = sm.stays(list(row), of(temperature, 1.0), of(top_k, 0), of(top_p, 1.0), of(min_p, 0.0))
            if sm.clear_of_borders(weights, random[i].item()):
                assert token[i].item() == sm.choose(weights, random[i].item())[0]
        self.count("sample")


@pytest.mark.parametrize("bits", [4, 8])
def test_every_call_of_a_run(monkeypatch, bits):
    from paper_2412_15803_amd import stream_decode as sd
    from paper_2412_15803_amd import wq

    announce(f"decoder of microscaled weights, {bits} bits")
    model = sd.MxDecoder(bits)
    checked = Checked(wq)
    monkeypatch.setattr(sd, "wq", checked)
    rng = np.random.default_rng(bits)
    prompts = [rng.integers(0, model.vocab, n).tolist() for n in (5, 90, 33)]
    allowed = torch.full((1, -(-model.vocab // 32)), 0x7FFF7FFF, dtype=torch.int32, device="cuda")
    steps = 4
    history, lens, _, _ = sd.generate(model, prompts, 2, steps, 40, 4, 16, allowed, sampler=sd.Sampler(0.8, top_k=50, top_p=0.95, min_p=0.01))
    for i, words in enumerate(history.tolist()):
        made = words[int(lens[i]) - steps:int(lens[i])]
        assert all(w % 32 not in (15, 31) for w in made)
    passes = steps + 1
    assert checked.calls == dict(norm=passes * 5, quantize=passes * 2, gated=passes * 2, linear=passes * 9, sample=steps)


def test_the_same_seed_gives_the_same_words():
    from paper_2412_15803_amd import stream_decode as sd

    model = sd.MxDecoder(8)
    prompts = [[1, 2, 3], list(range(40))]
    runs = [sd.generate(model, prompts, 3, 24, 40, 4, sampler=sd.Sampler(1.0, top_p=0.9, seed=seed))[0] for seed in (5, 5, 6)]
    assert torch.equal(runs[0], runs[1]) and not torch.equal(runs[0], runs[2])
    best = [sd.generate(model, prompts, 1, 24, 40, 4, sampler=sampler)[0] for sampler in (None, sd.Sampler(0.0, seed=1))]
    assert torch.equal(*best)  # a temperature of 0 takes the best words


def test_a_layer_captured_and_replayed():
    """Norm, linears, gated product, norm, logits and the next word in one graph, replayed with the program's own work between
    the replays."""
    from paper_2412_15803_amd import wq

    rows, hidden, inter, vocab = 40, 512, 1056, 3001
    g = torch.Generator(device="cuda").manual_seed(3)
    weights = []
    for n, k in ((2 * inter, hidden), (hidden, inter), (vocab, hidden)):
        w = wq.mx_empty(n, k, 4)
        wq.mx_quantize(torch.randn((n, k), generator=g, device="cuda") / math.sqrt(k), *w)
        weights.append(w)
    x = torch.zeros((rows, hidden), dtype=torch.bfloat16, device="cuda")
    more, total, gain = torch.zeros_like(x), torch.zeros_like(x), torch.ones(hidden, dtype=torch.bfloat16, device="cuda")
    a, b, c = wq.mx_empty(rows, hidden, 8), wq.mx_empty(rows, inter, 4), wq.mx_empty(rows, hidden, 8)
    gate_up, down = torch.empty((rows, 2 * inter), dtype=torch.bfloat16, device="cuda"), torch.empty_like(x)
    logits = torch.empty((rows, vocab), dtype=torch.bfloat16, device="cuda")
    random, top_p = torch.zeros(rows, device="cuda"), torch.full((rows,), 0.9, device="cuda")
    token, share = torch.zeros(rows, dtype=torch.int32, device="cuda"), torch.zeros(rows, device="cuda")
    pairs = ((weights[0][0], a[0]), (weights[1][0], b[0]), (weights[2][0], c[0]))
    linear_spaces, sample_space = [wq.mx_linear_workspace(*p) for p in pairs], wq.sample_workspace(logits)

    def step():
        wq.add_rmsnorm(x, gain, 1e-5, residual=more, total=total, codes=a[0], scales=a[1])
        wq.mx_linear(*weights[0], *a, gate_up, workspace=linear_spaces[0])
        wq.mx_quantize(gate_up, *b, gated=True)
        wq.mx_linear(*weights[1], *b, down, workspace=linear_spaces[1])
        wq.add_rmsnorm(total, gain, 1e-5, residual=down, codes=c[0], scales=c[1])
        wq.mx_linear(*weights[2], *c, logits, workspace=linear_spaces[2])
        wq.process_logits(logits, logits)
        wq.sample_logits(logits, random, token, top_p=top_p, share=share, workspace=sample_space)

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in range(4):
        g.manual_seed(seed)
        x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
        more.copy_(torch.randn(x.shape, generator=g, device="cuda"))
        random.copy_(torch.rand(rows, generator=g, device="cuda"))
        outputs = total, gate_up, down, logits, token, share
        for t in outputs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        kept = [t.clone() for t in outputs]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(kept, outputs))
        assert bool((token >= 0).all()) and float(logits.float().std()) > 0.1
