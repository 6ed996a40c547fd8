"""Microscaled matrices, the norm and the choice of words where offsets pass 32 bits."""

import math

import pytest
import torch

from gpu_util import announce, require_gpu
from paper_2412_15803_amd import wq

pytestmark = pytest.mark.gpu
APART = 1 << 31  # elements between two rows: the third row's begin 2^32 elements, 2^33 bytes, on


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    require_gpu()
    yield
    torch.cuda.empty_cache()


def rows_apart(cols, value):
    base = torch.empty(2 * APART + cols, dtype=torch.float16, device="cuda")
    t = base.as_strided((3, cols), (APART, 1))
    t.copy_(value)
    return t


def random(*shape, seed=1):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").half()


def same(a, b):
    return torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def used(scales, cols):
    return scales.view(torch.uint8)[:, :cols // 32]


def test_rows_far_apart():
    near = random(3, 512)
    far = rows_apart(512, near)
    for gated in (False, True):
        cols = 256 if gated else 512
        a, b = wq.mx_empty(3, cols, 8), wq.mx_empty(3, cols, 8)
        wq.mx_quantize(near, *a, gated=gated)
        wq.mx_quantize(far, *b, gated=gated)
        assert same(a[0], b[0]) and torch.equal(used(a[1], cols), used(b[1], cols))
    out, want = rows_apart(512, torch.zeros_like(near)), torch.empty_like(near)
    a = wq.mx_empty(3, 512, 4)
    wq.mx_quantize(near, *a)
    wq.mx_dequantize(*a, out)
    wq.mx_dequantize(*a, want)
    assert torch.equal(out, want)
    weight = random(512, seed=2)
    wq.add_rmsnorm(near, weight, 1e-5, out=want)
    wq.add_rmsnorm(far, weight, 1e-5, out=out)
    assert torch.equal(out, want)
    w, x = wq.mx_empty(512, 512, 4), wq.mx_empty(3, 512, 8)
    wq.mx_quantize(random(512, 512, seed=3), *w)
    wq.mx_quantize(near, *x)
    wq.mx_linear(*w, *x, want)
    wq.mx_linear(*w, *x, out)
    assert torch.equal(out, want)
    u, p = torch.tensor([0.1, 0.5, 0.9], device="cuda"), torch.full((3,), 0.9, device="cuda")
    token, other = (torch.empty(3, dtype=torch.int32, device="cuda") for _ in range(2))
    wq.sample_logits(near, u, token, top_p=p)
    wq.sample_logits(far, u, other, top_p=p)
    assert torch.equal(token, other)


def test_more_pieces_than_a_launch_takes():
    """2^31 pieces and more: two launches, codes beyond 2^32 bytes."""
    rows, cols = 16400, 1 << 20
    announce(f"quantize {rows} x {cols}")
    x = torch.empty((rows, cols), dtype=torch.float16, device="cuda")
    for i in range(0, rows, 1024):
        x[i:i + 1024].uniform_(-2, 2)
    codes, scales = wq.mx_empty(rows, cols, 4)
    wq.mx_quantize(x, codes, scales)
    some = [0, 4095, 4096, 8191, 8192, 16382, 16383, 16384, rows - 1]
    for i in some:
        c, s = wq.mx_empty(1, cols, 4)
        wq.mx_quantize(x[i:i + 1], c, s)
        assert same(c, codes[i:i + 1]) and torch.equal(used(s, cols), used(scales, cols)[i:i + 1]), i
    want = torch.empty((1, cols), dtype=torch.float16, device="cuda")
    wq.mx_dequantize(codes, scales, x)
    for i in some:
        wq.mx_dequantize(codes[i:i + 1], scales[i:i + 1], want)
        assert torch.equal(want, x[i:i + 1]), i


@pytest.mark.parametrize("n,k,m", [((1 << 17) + 16, 65536, 3), ((1 << 17) + 16, 65536, 20), ((1 << 17) + 16, 65536, 70), (20, 32768, (1 << 17) + 16), (300, 32768, (1 << 17) + 16)])
def test_linears_of_large_matrices(n, k, m):
    """Codes of W or of x beyond 2^32 bytes: the ends of the result against float64."""
    announce(f"linear {n} x {k}, {m} rows")
    w, x = wq.mx_empty(n, k, 4), wq.mx_empty(m, k, 8)
    for (codes, scales), bits in ((w, 4), (x, 8)):
        step = max(1, (1 << 28) // k)
        for i in range(0, codes.shape[0], step):
            part = codes[i:i + step].view(torch.uint8)
            part.random_(0, 256 if bits == 4 else 0x50)
        scales.view(torch.uint8).random_(122, 128)
    y = torch.empty((m, n), dtype=torch.bfloat16, device="cuda")
    wq.mx_linear(*w, *x, y)

    def ends(codes, scales):
        rows = codes.shape[0]
        at = torch.tensor(sorted({0, rows // 2, max(rows - 17, 0), max(rows - 3, 0), rows - 1}), device="cuda")
        out = torch.empty((len(at), k), device="cuda")
        wq.mx_dequantize(codes.view(torch.uint8)[at].view(codes.dtype), scales.view(torch.uint8)[at], out)
        return at, out.double()

    (ni, wv), (mi, xv) = ends(*w), ends(*x)
    want, weight = xv @ wv.t().contiguous(), xv.abs() @ wv.abs().t().contiguous()
    off = (y[mi][:, ni].double() - want).abs() - (2.0 ** -8 * want.abs() + 2.0 ** -13 * weight + 2.0 ** -126)
    assert bool((off <= 0).all()), float(off.max())
    assert math.isfinite(float(want.abs().max()))
