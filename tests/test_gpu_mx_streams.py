"""The norm, rounding, linears and the choice of words on streams other than the current one, several at once."""

import pytest
import torch

from gpu_util import require_gpu
from paper_2412_15803_amd import wq

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    require_gpu()


class Work:
    """One chain of all operators on inputs of its own."""

    def __init__(self, seed, rows=40, hidden=1024, vocab=20011):
        g = torch.Generator(device="cuda").manual_seed(seed)
        randn = lambda *shape: torch.randn(shape, generator=g, device="cuda").half()  # noqa: E731
        self.source, self.more, self.gain = randn(rows, hidden), randn(rows, hidden), randn(hidden)
        self.w = wq.mx_empty(vocab, hidden // 2, 4)
        wq.mx_quantize(randn(vocab, hidden // 2) / 16, *self.w)
        self.x, self.normed = torch.zeros_like(self.source), torch.zeros_like(self.source)
        self.a = wq.mx_empty(rows, hidden // 2, 8)
        self.logits = torch.zeros((rows, vocab), dtype=torch.float16, device="cuda")
        self.random, self.top_p = torch.rand(rows, generator=g, device="cuda"), torch.full((rows,), 0.9, device="cuda")
        self.token, self.share = torch.zeros(rows, dtype=torch.int32, device="cuda"), torch.zeros(rows, device="cuda")

    def run(self, stream=None):
        on = dict(stream=stream)
        wq.add_rmsnorm(self.x, self.gain, 1e-5, out=self.normed, residual=self.more, total=self.x, **on)
        wq.mx_quantize(self.normed, *self.a, gated=True, **on)
        wq.mx_linear(*self.w, *self.a, self.logits, **on)
        wq.sample_logits(self.logits, self.random, self.token, top_p=self.top_p, share=self.share, **on)

    def outputs(self):
        return [t.clone() for t in (self.x, self.normed, self.logits, self.token, self.share)]


def test_streams_at_once():
    """Workspaces made in the calls, inputs that are ready on the call's stream only."""
    works = [Work(seed) for seed in range(3)]
    want = []
    for w in works:
        w.x.copy_(w.source)
        w.run()
        want.append(w.outputs())
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in works]
    busy = [torch.randn((2048, 2048), device="cuda") for _ in works]
    torch.cuda.synchronize()
    for _ in range(5):
        for w, s, b in zip(works, streams, busy):
            with torch.cuda.stream(s):
                for t in (w.normed, w.logits, w.token, w.share):
                    t.zero_()
                w.x.copy_(w.source + 0 * (b @ b)[:40, :1024].half().nan_to_num(0, 0, 0))  # (late)
            w.run(stream=s)
        torch.cuda.synchronize()
        for w, expected in zip(works, want):
            assert all(torch.equal(a, b) for a, b in zip(w.outputs(), expected))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
def test_sum_and_norm_in_the_inputs_places(dtype):
    g = torch.Generator(device="cuda").manual_seed(2)
    x, r = (torch.randn((50, 2080), generator=g, device="cuda").to(dtype) for _ in range(2))
    gain = torch.randn(2080, generator=g, device="cuda").to(dtype)
    total, out = torch.empty_like(x), torch.empty_like(x)
    wq.add_rmsnorm(x, gain, 1e-5, out=out, residual=r, total=total)
    for places in ((0, 1), (1, 0)):
        held = [x.clone(), r.clone()]
        wq.add_rmsnorm(held[0], gain, 1e-5, total=held[places[0]], out=held[places[1]], residual=held[1])
        assert torch.equal(held[places[0]], total) and torch.equal(held[places[1]], out)
