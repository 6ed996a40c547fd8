"""y = x W^T of microscaled matrices on the GPU against float64: every shape of tile with rows of every length
around its stages, in parts of K and whole."""

import numpy as np
import pytest
import torch

import mx_gpu as mg
import mx_model as mm
from gpu_util import require_gpu
from paper_2412_15803_amd import wq
from test_gpu_mx_linear import assert_close, run

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    require_gpu()


LENGTHS = [32, 96, 128, 160, 224, 256, 288, 480, 512, 544, 736, 768, 800, 1056, 1504, 2048, 2080, 3616, 4128]


def check(seed, n, k, m, bits, dtype, pad=0):
    rng = np.random.default_rng(seed)
    w, ws = mg.random_matrix(rng, n, k, 4, 124, 130)
    x, xs = mg.random_matrix(rng, m, k, bits, 124, 130)
    if bits == 8:
        x = ((x & 0x87) | (rng.integers(4, 9, x.shape).astype(np.uint8) << 3)).astype(np.uint8)
    got = run((w, ws), (x, xs), bits, n, m, dtype, pad=pad)
    wv, xv = torch.from_numpy(mm.values(w, ws, 4)).cuda(), torch.from_numpy(mm.values(x, xs, bits)).cuda()
    want, weight = xv @ wv.t().contiguous(), xv.abs() @ wv.abs().t().contiguous()
    assert_close(got, want.cpu().numpy(), weight.cpu().numpy(), dtype)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("k", LENGTHS)
def test_small_tiles(bits, k):
    """Up to 32 rows, up to 64, and more: a workgroup to each CU at most."""
    check(k, 70, k, 17 + k % 16, bits, torch.float16, pad=2)
    check(k, 129, k, 33 + k % 32, bits, torch.bfloat16, pad=8)
    check(k, 200, k, 66, bits, torch.float16)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("k", [96, 256, 288, 544, 1056])
def test_more_tiles_than_cus(bits, k):
    check(k, 16500, k, 20, bits, torch.float16, pad=4)
    check(k, 16500, k, 50, bits, torch.float16, pad=4)
    check(k, 4100, k, 300, bits, torch.bfloat16, pad=4)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("k", [32, 160, 256, 288, 480, 544, 800])
def test_larger_tiles(bits, k):
    check(k, 3300, k, 1100, bits, torch.float16, pad=4)
    check(k, 3601, k, 3585, bits, torch.bfloat16, pad=7)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("n,m", [(48, 5), (48, 40), (4100, 300)])
def test_sums_of_products_below_the_normal_numbers(bits, n, m):
    """128 products of 2^-135 and 2^-134 at a time, whose sums are normal numbers only together."""
    k = 8192
    w, ws = np.full((n, k), 2, dtype=np.uint8), np.full((n, k // 32), 60, dtype=np.uint8)  # 1 x 2^-67
    x, xs = np.full((m, k), 2 if bits == 4 else 0x38, dtype=np.uint8), np.full((m, k // 32), 59, dtype=np.uint8)  # 1 x 2^-68
    w[1::2] = 4
    got = run((w, ws), (x, xs), bits, n, m, torch.bfloat16)
    wv, xv = mm.values(w, ws, 4), mm.values(x, xs, bits)
    assert_close(got, xv @ wv.T, np.abs(xv) @ np.abs(wv).T, torch.bfloat16)


def test_two_streams_with_workspaces_of_their_own():
    """The same linear in parts of K on two streams at once, and captured for both."""
    rng = np.random.default_rng(1)
    n, k, m = 300, 4096, 40
    w, ws = mg.random_matrix(rng, n, k, 4, 124, 130)
    wd = mg.to_device(w, ws, 4)
    xs = [mg.to_device(*mg.random_matrix(rng, m, k, 8, 124, 130), 8) for _ in range(2)]
    assert wq.mx_linear_workspace_size(n, k, m, 8) > 0
    want = []
    for x in xs:
        y = torch.empty((m, n), dtype=torch.float16, device="cuda")
        wq.mx_linear(*wd, *x, y)
        want.append(y)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    spaces = [wq.mx_linear_workspace(wd[0], x[0]) for x in xs]
    got = [torch.zeros_like(y) for y in want]
    for _ in range(20):
        for i, s in enumerate(streams):
            wq.mx_linear(*wd, *xs[i], got[i], workspace=spaces[i], stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graphs = []
    for i, s in enumerate(streams):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            wq.mx_linear(*wd, *xs[i], got[i], workspace=spaces[i])
        graphs.append(graph)
    for _ in range(3):
        for y in got:
            y.zero_()
        torch.cuda.synchronize()
        for s, graph in zip(streams, graphs):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
