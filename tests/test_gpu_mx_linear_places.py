"""y = x W^T of microscaled matrices: every element in its place, at up to 16 rows and in tiles of 128 and 256; up to
16 rows with more workgroups than CUs; which calls give the same bits."""

import numpy as np
import pytest
import torch

import mx_gpu as mg
import mx_model as mm
from gpu_util import require_gpu
from paper_2412_15803_amd import wq
from test_gpu_mx_linear import case, run
from test_gpu_mx_linear_bounds import assert_within

pytestmark = pytest.mark.gpu
TYPES = [torch.float16, torch.bfloat16]


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    require_gpu()


def tiles(n, m, side):
    return -(-n // side) * -(-m // side)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("n,k,m", [(48, 672, 16), (4200, 2080, 2), (4200, 2080, 4), (4200, 2080, 8), (4200, 14336, 16), (24600, 672, 70), (49100, 672, 130)])
def test_every_element_finds_its_place(bits, n, k, m):
    """One element of x in each row, in another column each, until all columns had one: the output is that column of
    w, exactly."""
    if m > 16:  # the tiles that these sizes are meant for
        side = 128 if m < 128 else 256
        assert m > side // 2 and tiles(n, m, side) >= 192 and (m <= 128 or side == 256)
    rng = np.random.default_rng(bits)
    w, ws = mg.random_matrix(rng, n, k, 4, 120, 134)
    wd = mg.to_device(w, ws, 4)
    wv = torch.empty((n, k), dtype=torch.bfloat16, device="cuda")  # (E2M1 values under these scales are exact.)
    wq.mx_dequantize(*wd, wv)
    assert np.array_equal(wv[:50].double().cpu().numpy(), mm.values(w[:50], ws[:50], 4))
    wv = wv.t().contiguous()
    rows = torch.arange(m, device="cuda")
    x = torch.zeros((m, k if bits == 8 else k // 2), dtype=torch.uint8, device="cuda")
    xs = torch.full((m, mm.stride(k)), 255, dtype=torch.uint8, device="cuda")
    y = torch.empty((m, n), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(bits)
    for first in range(0, k, m):
        at = (first + rows) % k
        xs[:, :k // 32] = torch.randint(124, 131, (m, k // 32), generator=g, device="cuda", dtype=torch.uint8)
        x.zero_()
        if bits == 8:
            x[rows, at] = 0x38
        else:
            x[rows, at // 2] = torch.where(at % 2 == 1, 0x20, 0x02).to(torch.uint8)
        wq.mx_linear(*wd, x.view(torch.float8_e4m3fn) if bits == 8 else x, xs, y)
        want = wv[at] * torch.exp2(xs[rows, at // 32].float() - 127).to(torch.bfloat16)[:, None]
        assert torch.equal(y, want), (first, (y != want).nonzero()[:4].tolist())


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("n,k", [(4100, 544), (4113, 4096), (4100, 7200), (8209, 96)])
@pytest.mark.parametrize("m", [1, 2, 3, 5, 8, 9, 16])
def test_few_rows_of_many_outputs(bits, n, k, m):
    """More than 256 workgroups, whose waves are as many as leave room for others beside them."""
    assert -(-n // 16) > 256 and m <= 16
    w, x, want, weight = case(np.random.default_rng(n + k + m), n, k, m, bits)
    want, weight = torch.from_numpy(want).cuda(), torch.from_numpy(weight).cuda()
    for dtype in TYPES:
        assert_within(run(w, x, bits, n, m, dtype, pad=m % 3), want, weight, k, bits, dtype)


@pytest.mark.parametrize("bits", [4, 8])
def test_the_same_call_gives_the_same_bits(bits):
    """Again and again, in a graph too; a row among more or fewer others lies within the bound, with the same bits
    where as many rows share LDS (up to 2, 4, 8 and 16)."""
    n, k = 4200, 14336
    rng = np.random.default_rng(3)
    w, x, want, weight = case(rng, n, k, 40, bits)
    wd, xd = mg.to_device(*w, 4), mg.to_device(*x, bits)
    want, weight = torch.from_numpy(want).cuda(), torch.from_numpy(weight).cuda()
    results = {}
    for m in (1, 2, 3, 4, 6, 8, 9, 16, 17, 33, 40):
        y, again = (torch.empty((m, n), dtype=torch.float16, device="cuda") for _ in range(2))
        part = xd[0][:m], xd[1][:m]
        wq.mx_linear(*wd, *part, y)
        for _ in range(3):
            again.zero_()
            wq.mx_linear(*wd, *part, again)
            assert torch.equal(y, again)
        graph = torch.cuda.CUDAGraph()
        workspace = wq.mx_linear_workspace(wd[0], part[0])
        with torch.cuda.graph(graph):
            wq.mx_linear(*wd, *part, again, workspace=workspace)
        for _ in range(2):
            again.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, again)
        assert_within(y, want[:m], weight[:m], k, bits, torch.float16)
        results[m] = y
    for fewer, more in ((1, 2), (3, 4), (6, 8), (9, 16)):
        assert torch.equal(results[fewer], results[more][:fewer])
