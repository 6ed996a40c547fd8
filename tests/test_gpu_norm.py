"""The residual's addition and the norm on the GPU against float64."""

import numpy as np
import pytest
import torch

import mx_gpu as mg
import mx_model as mm
from gpu_util import require_gpu
from paper_2412_15803_amd import wq

pytestmark = pytest.mark.gpu
TYPES = [torch.float16, torch.bfloat16, torch.float32]
# fp32 sums of squares: a lane adds 32 at most, then six steps of a wave and 16 of the block: below 60 roundings of 2^-24,
# halved by the root; the root, the quotients and products, and the sum of x and the residual add six more.
REL = 2.0 ** -18


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    require_gpu()


def model(x, residual, weight, eps):
    s = x.double() + (residual.double() if residual is not None else 0)
    return s, s / torch.sqrt(s.square().mean(-1, keepdim=True) + eps) * weight.double()


def assert_rounded(got, want, dtype, rel):
    """`got` is `want`, known to `rel`, rounded once to dtype."""
    info = torch.finfo(dtype)
    bound = want.abs() * (info.eps / 2 + rel) * (1 + rel) + info.tiny * info.eps / 2 + 1e-45
    assert bool(((got.double() - want).abs() <= bound).all()), float(((got.double() - want).abs() / bound).max())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,dim,pad,residual", [(1, 32, 0, True), (1, 4096, 0, True), (77, 2080, 0, False), (5, 96, 8, True), (3, 8224, 0, True), (2, 16416, 24, True),
                                                   (2, 32768, 0, False), (300, 512, 0, True), (1000, 1024, 0, False)])
def test_norm(dtype, rows, dim, pad, residual):
    g = torch.Generator(device="cuda").manual_seed(rows * dim)
    make = lambda: (torch.randn((rows, dim + pad), generator=g, device="cuda") * 2).to(dtype)[:, :dim]  # noqa: E731
    x, r = make(), make() if residual else None
    weight = (torch.randn(dim, generator=g, device="cuda") * 0.2 + 1).to(dtype)
    total, out = (torch.full((rows, dim + pad), 5.0, dtype=dtype, device="cuda") for _ in range(2))
    s, v = model(x, r, weight, 1e-5)
    for bits in (4, 8):
        codes, scales = mg.room(rows, dim, bits)
        wq.add_rmsnorm(x, weight, 1e-5, out=out[:, :dim], residual=r, total=total[:, :dim], codes=codes, scales=scales)
        assert_rounded(total[:, :dim], s, dtype, 2.0 ** -24)
        assert_rounded(out[:, :dim], v, dtype, REL)
        c, sc, padding = mg.to_host(codes, scales, bits)
        mm.check_rounded(c, sc, v.cpu().numpy(), bits, REL)
        assert np.all(padding == 0xA5)
    if pad:
        assert bool((total[:, dim:] == 5).all()) and bool((out[:, dim:] == 5).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_outputs_alone_and_in_place(dtype):
    """Each output alone is what it is beside the others, and may take an input's place."""
    g = torch.Generator(device="cuda").manual_seed(1)
    x, r = (torch.randn((9, 1056), generator=g, device="cuda").to(dtype) for _ in range(2))
    weight = torch.ones(1056, dtype=dtype, device="cuda")
    total, out = torch.empty_like(x), torch.empty_like(x)
    codes, scales = mg.room(9, 1056, 8)
    wq.add_rmsnorm(x, weight, 1e-6, out=out, residual=r, total=total, codes=codes, scales=scales)
    alone = torch.empty_like(x)
    wq.add_rmsnorm(x, weight, 1e-6, out=alone, residual=r)
    assert torch.equal(alone, out)
    c, s = mg.room(9, 1056, 8)
    wq.add_rmsnorm(x, weight, 1e-6, residual=r, codes=c, scales=s)
    assert torch.equal(c.view(torch.uint8), codes.view(torch.uint8)) and torch.equal(s.view(torch.uint8), scales.view(torch.uint8))
    xx, rr = x.clone(), r.clone()
    wq.add_rmsnorm(xx, weight, 1e-6, out=xx, residual=rr, total=rr)
    assert torch.equal(xx, out) and torch.equal(rr, total)
    xx = x.clone()
    wq.add_rmsnorm(xx, weight, 1e-6, out=alone, residual=xx, total=xx)
    twice = torch.empty_like(x)
    wq.add_rmsnorm(x, weight, 1e-6, out=twice, residual=x, total=total)
    assert torch.equal(alone, twice) and torch.equal(xx, total)


def test_zero_rows_and_values_that_are_none():
    x = torch.randn((5, 64), device="cuda")
    x[1] = 0
    x[2, 40] = float("nan")
    x[3, 3] = float("inf")
    weight = torch.ones(64, device="cuda")
    out = torch.empty_like(x)
    codes, scales = mg.room(5, 64, 8)
    wq.add_rmsnorm(x, weight, 1e-5, out=out, codes=codes, scales=scales)
    _, s, _ = mg.to_host(codes, scales, 8)
    assert bool((out[1] == 0).all()) and np.all(s[1] == 0)
    assert bool(torch.isnan(out[2]).all()) and np.all(s[2] == 255)
    # Infinity over infinity in its own place, finite values over it elsewhere.
    assert bool(torch.isnan(out[3, 3])) and bool((out[3, 4:] == 0).all()) and s[3, 0] == 255 and s[3, 1] == 0
    assert bool(torch.isfinite(out[[0, 4]]).all())
    wq.add_rmsnorm(x[1:2], weight, 0.0, out=out[1:2])
    assert bool(torch.isnan(out[1]).all())  # 0 / 0


def test_captured_and_replayed():
    x = torch.zeros((65, 2080), dtype=torch.float16, device="cuda")
    r, out, total = torch.ones_like(x), torch.empty_like(x), torch.empty_like(x)
    weight = torch.ones(2080, dtype=torch.float16, device="cuda")
    codes, scales = mg.room(65, 2080, 4)

    def step():
        wq.add_rmsnorm(x, weight, 1e-5, out=out, residual=r, total=total, codes=codes, scales=scales)

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in range(3):
        x.copy_(torch.randn(x.shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        kept = [t.clone() for t in (out, total, codes, scales.view(torch.uint8)[:, :65])]
        step()
        assert all(torch.equal(a, b) for a, b in zip(kept, (out, total, codes, scales.view(torch.uint8)[:, :65])))
