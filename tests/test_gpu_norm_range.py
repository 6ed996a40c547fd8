"""The norm of rows whose squares leave fp32's range, against float64 and the bound of include/wq_norm.h."""

import numpy as np
import pytest
import torch

import mx_gpu as mg
import mx_model as mm
from gpu_util import require_gpu
from paper_2412_15803_amd import wq

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    require_gpu()


def check(x, weight, eps, residual=None):
    """All outputs of x + residual, which is exact in fp32."""
    rows, dim = x.shape
    dtype = x.dtype
    info = torch.finfo(dtype)
    s = x.double() + (residual.double() if residual is not None else 0)
    assert torch.equal(s, s.float().double())
    eps = float(np.float32(eps))
    w = weight.double()
    v = s / torch.sqrt(s.square().mean(-1, keepdim=True) + eps) * w
    known = 2.0 ** -18 * v.abs() + 2.0 ** -149 * (1 + w.abs())
    # One rounding to dtype of a value that is known so: half a step, of the smallest normal number's steps at least.
    bound = known + (v.abs() + known) * info.eps / 2 + info.tiny * info.eps / 2
    out, total = torch.empty_like(x), torch.empty_like(x)
    for bits in (4, 8):
        codes, scales = mg.room(rows, dim, bits)
        wq.add_rmsnorm(x, weight, eps, out=out, residual=residual, total=total, codes=codes, scales=scales)
        assert torch.equal(total, s.to(dtype))
        off = (out.double() - v).abs()
        assert bool((off <= bound).all()), float((off / bound).max())
        c, sc, _ = mg.to_host(codes, scales, bits)
        # (Nothing here has a v so small that the absolute part of the bound counts in a block's scale.)
        mm.check_rounded(c, sc, v.cpu().numpy(), bits, 2.0 ** -17)


# Lanes with one piece, with two and with four.
DIMS = [32, 4096, 8224, 16416, 32768]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("eps", [0.0, 1e-45, 1e-38, 1e-30])
def test_small_rows(dtype, dim, eps):
    """Squares that vanish, and squares with few digits left."""
    g = torch.Generator(device="cuda").manual_seed(dim)
    e = torch.tensor([-18, -19, -20, -21, -22, -23, -25, -30, -34], device="cuda", dtype=torch.float64)[:, None]
    x = (torch.randn((len(e), dim), generator=g, device="cuda", dtype=torch.float64) * 10.0 ** e).to(dtype)
    weight = (torch.randn(dim, generator=g, device="cuda") * 0.2 + 1).to(dtype)
    check(x, weight, eps)


@pytest.mark.parametrize("dim", DIMS)
def test_denormal_rows(dim):
    """Rows of fp32's smallest numbers; one of them alone among zeros."""
    g = torch.Generator(device="cuda").manual_seed(dim)
    x = torch.randint(-3, 4, (4, dim), generator=g, device="cuda").double()
    x[1] *= 1000.0
    x[2] = 0
    x[2, dim - 5] = 1.0
    x[3] = 0
    x[3, 3] = -7.0
    x = (x * 2.0 ** -149).float()
    weight = torch.randn(dim, generator=g, device="cuda")
    for eps in (0.0, 1e-45, 1e-42):
        check(x, weight, eps)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("eps", [0.0, 1e-5, 3e38])
def test_large_rows(dtype, dim, eps):
    """Sums of squares, and squares, that pass fp32's largest number."""
    g = torch.Generator(device="cuda").manual_seed(dim)
    e = torch.tensor([17, 18, 19, 20, 30, 37], device="cuda", dtype=torch.float64)[:, None]
    x = (torch.randn((len(e), dim), generator=g, device="cuda", dtype=torch.float64) * 10.0 ** e).to(dtype)
    x[0, 0] = 2.0 ** 100
    weight = (torch.randn(dim, generator=g, device="cuda") * 0.2 + 1).to(dtype)
    check(x, weight, eps)


def test_beside_ordinary_rows_with_a_residual_and_in_place():
    """A row's way is its own: the rows around it keep their bits."""
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn((7, 2080), generator=g, device="cuda")
    weight = torch.randn(2080, generator=g, device="cuda")
    plain = torch.empty_like(x)
    wq.add_rmsnorm(x, weight, 1e-6, out=plain)
    x[1] *= 2.0 ** -100
    x[4] *= 2.0 ** 90
    check(x, weight, 1e-6, residual=x)
    out = torch.empty_like(x)
    wq.add_rmsnorm(x, weight, 1e-6, out=out)
    ordinary = [0, 2, 3, 5, 6]
    assert torch.equal(out[ordinary], plain[ordinary])
    wq.add_rmsnorm(x, weight, 1e-6, out=x)
    assert torch.equal(x, out)


def test_rows_of_values_that_are_none():
    """What the header says of zeros without eps, infinities and NaN."""
    x = torch.full((5, 96), 1e30, device="cuda")
    x[0] = 0
    x[1, 40], x[2, 40] = float("inf"), float("nan")
    x[3, 7], x[3, 8] = float("inf"), float("-inf")
    x[4] = 1e-30
    x[4, 95] = float("inf")
    weight, out = torch.ones(96, device="cuda"), torch.empty_like(x)
    wq.add_rmsnorm(x, weight, 0.0, out=out)
    assert bool(torch.isnan(out[0]).all()) and bool(torch.isnan(out[2]).all())
    for row, places in ((1, [40]), (3, [7, 8]), (4, [95])):
        bad = torch.zeros(96, dtype=torch.bool, device="cuda")
        bad[places] = True
        assert torch.equal(torch.isnan(out[row]), bad) and bool((out[row][~bad] == 0).all())
