"""The bound of include/wq_mx.h where the matrix cores leave out most: large products beside small ones that they
cancel, and long sums of one sign behind a large beginning."""

import numpy as np
import pytest
import torch

import mx_gpu as mg
import mx_model as mm
from gpu_util import require_gpu
from paper_2412_15803_amd import wq
from test_gpu_mx_linear import run

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    require_gpu()


def assert_within(got, want, weight, k, bits, dtype):
    info = torch.finfo(dtype)
    bound = info.eps / 2 * want.abs() + ((2.0 ** -9 if bits == 8 else 2.0 ** -15) + k * 2.0 ** -26) * weight + (2.0 ** -25 if dtype is torch.float16 else 2.0 ** -126)
    off = (got.double() - want).abs() / bound
    assert bool((off <= 1).all()), float(off.max())


SIZES = [(48, 672, 5), (48, 672, 30), (100, 4096, 40), (4128, 288, 16), (3300, 544, 1100), (3601, 160, 3585)]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("large_w,large_x,small_x", [(2, 0x7E, 0x0E), (1, 0x78, 0x0F), (7, 0x78, 0x17), (3, 0x7E, 0x0A)])
@pytest.mark.parametrize("n,k,m", SIZES)
def test_large_products_that_cancel(dtype, large_w, large_x, small_x, n, k, m):
    """Of each eight products one is large, the other seven of one sign and 2^-13 to 2^-15 of it; the next eight have
    the same large one with the other sign."""
    rng = np.random.default_rng(n + large_w)
    w, x = np.full((n, k), 2, dtype=np.uint8), np.full((m, k), small_x, dtype=np.uint8)
    at = rng.integers(0, 8, k // 8)
    at[1::2] = at[0::2]
    places = np.arange(0, k, 8) + at
    w[:, places] = large_w
    x[:, places] = large_x
    x[:, places[1::2]] |= 0x80
    x[1::2] ^= 0x80
    w[rng.random((n, 1)).repeat(k, 1) < 0.3] |= 8
    ws, xs = np.full((n, k // 32), 127, dtype=np.uint8), np.full((m, k // 32), 127, dtype=np.uint8)
    got = run((w, ws), (x, xs), 8, n, m, dtype)
    wv, xv = torch.from_numpy(mm.values(w, ws, 4)).cuda(), torch.from_numpy(mm.values(x, xs, 8)).cuda()
    assert_within(got, xv @ wv.t().contiguous(), xv.abs() @ wv.abs().t().contiguous(), k, 8, dtype)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("spread", [0, 3, 12])
@pytest.mark.parametrize("n,k,m", SIZES)
def test_codes_of_every_size(bits, spread, n, k, m):
    """All codes alike often, and blocks whose scales are far apart."""
    rng = np.random.default_rng(k + spread)
    w, ws = mg.random_matrix(rng, n, k, 4, 127 - spread, 127 + spread)
    x, xs = mg.random_matrix(rng, m, k, bits, 127 - spread, 127 + spread)
    got = run((w, ws), (x, xs), bits, n, m, torch.bfloat16)
    wv, xv = torch.from_numpy(mm.values(w, ws, 4)).cuda(), torch.from_numpy(mm.values(x, xs, bits)).cuda()
    assert_within(got, xv @ wv.t().contiguous(), xv.abs() @ wv.abs().t().contiguous(), k, bits, torch.bfloat16)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("k", [1 << 14, 1 << 18, 1 << 20])
@pytest.mark.parametrize("n,m,parts", [(40, 3, False), (40, 100, True), (8256, 17, False)])
def test_long_sums_behind_a_large_beginning(bits, k, n, m, parts):
    """128 times 1.5, then products so small that eight to thirty-two of them are just below what is kept beside 192."""
    assert (wq.mx_linear_workspace_size(n, k, m, bits) > 0) == parts
    w = torch.full((n, k // 2), 0x22, dtype=torch.uint8, device="cuda")
    ws = torch.full((n, mm.stride(k)), 127, dtype=torch.uint8, device="cuda")
    x = torch.full((m, k // 2 if bits == 4 else k), 0x33 if bits == 4 else 0x3C, dtype=torch.uint8, device="cuda")
    xs = torch.empty((m, mm.stride(k)), dtype=torch.uint8, device="cuda")
    y = torch.empty((m, n), dtype=torch.float16, device="cuda")
    for e in range(-24, -18):
        xs[:, :4], xs[:, 4:] = 127, 127 + e
        wq.mx_linear(w, ws, x if bits == 4 else x.view(torch.float8_e4m3fn), xs, y)
        want = torch.full((m, n), 192 + (k - 128) * 1.5 * 2.0 ** e, dtype=torch.float64, device="cuda")
        assert_within(y, want, want, k, bits, torch.float16)
