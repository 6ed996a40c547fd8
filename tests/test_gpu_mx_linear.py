"""y = x W^T of microscaled matrices on the GPU against float64."""

import numpy as np
import pytest
import torch

import mx_gpu as mg
import mx_model as mm
from gpu_util import require_gpu
from paper_2412_15803_amd import wq

pytestmark = pytest.mark.gpu
TYPES = [torch.float16, torch.bfloat16]


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    require_gpu()


def assert_close(got, want, weight, dtype):
    """The bound of include/wq_mx.h."""
    info = torch.finfo(dtype)
    got = got.double().cpu().numpy()
    bound = info.eps / 2 * np.abs(want) + 2.0 ** -13 * weight + (2.0 ** -25 if dtype is torch.float16 else 2.0 ** -126)
    off = np.abs(got - want) - bound
    assert np.all(off <= 0), (float(off.max()), np.unravel_index(off.argmax(), off.shape))


def case(rng, n, k, m, bits, low=124, high=130):
    w, ws = mg.random_matrix(rng, n, k, 4, low, high)
    x, xs = mg.random_matrix(rng, m, k, bits, low, high)
    if bits == 8:  # values of an activation: exponents of a few steps
        x = ((x & 0x87) | (rng.integers(4, 9, x.shape).astype(np.uint8) << 3)).astype(np.uint8)
    wv, xv = mm.values(w, ws, 4), mm.values(x, xs, bits)
    return (w, ws), (x, xs), xv @ wv.T, np.abs(xv) @ np.abs(wv).T


def run(w, x, bits, n, m, dtype, pad=0):
    wide = torch.full((m, n + pad), 7.0, dtype=dtype, device="cuda")
    wq.mx_linear(*mg.to_device(*w, 4), *mg.to_device(*x, bits), wide[:, :n])
    assert bool((wide[:, n:] == 7.0).all())
    return wide[:, :n]


SIZES = [(1, 32, 1), (16, 128, 16), (17, 512, 2), (3, 96, 5), (100, 160, 17), (250, 544, 33), (64, 2080, 48), (33, 1056, 49), (130, 4096, 64), (1003, 2080, 31),
         (16, 32, 65), (64, 64, 64), (65, 96, 66), (129, 160, 129), (200, 544, 300), (1003, 2080, 77), (64, 4096, 100), (4, 14336, 70), (2048, 512, 1), (40, 16384, 7)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("n,k,m", SIZES)
def test_sizes(dtype, bits, n, k, m):
    w, x, want, weight = case(np.random.default_rng(n + k + m), n, k, m, bits)
    assert_close(run(w, x, bits, n, m, dtype, pad=(n + m) % 3), want, weight, dtype)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("n,k,m", [(3600, 512, 3200), (3300, 672, 3400), (1536, 1024, 2100), (2100, 288, 1500), (4400, 96, 5000), (5000, 160, 4400), (4500, 288, 4600),
                                   (4700, 512, 4300), (4600, 544, 4353), (4354, 1184, 4700), (3000, 32, 3001), (3010, 256, 3000), (3000, 544, 2900), (2990, 640, 3030)])
def test_large_tiles(bits, n, k, m):
    """Sizes at which the larger tiles run and workgroups take several of them, ragged ones among them, from one
    step of K on; float64 on the GPU."""
    rng = np.random.default_rng(n)
    w, ws = mg.random_matrix(rng, n, k, 4, 124, 130)
    x, xs = mg.random_matrix(rng, m, k, bits, 124, 130)
    if bits == 8:
        x = ((x & 0x87) | (rng.integers(4, 9, x.shape).astype(np.uint8) << 3)).astype(np.uint8)
    got = run((w, ws), (x, xs), bits, n, m, torch.float16, pad=4)
    wv, xv = torch.from_numpy(mm.values(w, ws, 4)).cuda(), torch.from_numpy(mm.values(x, xs, bits)).cuda()
    want, weight = xv @ wv.t().contiguous(), xv.abs() @ wv.abs().t().contiguous()
    assert_close(got, want.cpu().numpy(), weight.cpu().numpy(), torch.float16)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("n,m", [(48, 20), (100, 90)])
def test_every_element_finds_its_place(bits, n, m):
    """One element of x at a time, its place shifted from row to row: the output is that
    column of w, exactly."""
    rng = np.random.default_rng(bits)
    k = 672
    w, ws = mg.random_matrix(rng, n, k, 4, 120, 134)
    wv = mm.values(w, ws, 4)
    one = 2 if bits == 4 else 0x38
    for first in range(0, k, m):
        x, xs = np.zeros((m, k), dtype=np.uint8), rng.integers(124, 131, (m, k // 32)).astype(np.uint8)
        at = (first + np.arange(m)) % k
        x[np.arange(m), at] = one
        got = run((w, ws), (x, xs), bits, n, m, torch.bfloat16).double().cpu().numpy()
        assert np.array_equal(got, wv[:, at].T * np.ldexp(1.0, xs[np.arange(m), at // 32].astype(int) - 127)[:, None])


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("n,k,m", [(20, 160, 3), (70, 672, 80)])
def test_nan_reaches_what_it_takes_part_in(bits, n, k, m):
    rng = np.random.default_rng(5)
    w, x, want, weight = case(rng, n, k, m, bits)
    w[1][4, k // 32 - 1] = 255
    x[1][2, 0] = 255
    if bits == 8:
        x[0][1, k - 1] = 0x7F
    got = run(w, x, bits, n, m, torch.float16)
    bad = np.zeros((m, n), dtype=bool)
    bad[:, 4] = bad[2] = True
    if bits == 8:
        bad[1] = True
    assert np.array_equal(torch.isnan(got).cpu().numpy(), bad)
    assert_close(torch.where(torch.from_numpy(bad).cuda(), torch.zeros_like(got), got), np.where(bad, 0, want), weight, torch.float16)


@pytest.mark.parametrize("n,k,m", [(32, 544, 5), (80, 544, 70)])
def test_scales_over_their_range(n, k, m):
    """Scales from 2^-127 to 2^127 whose products are ordinary, and ones that overflow or vanish."""
    rng = np.random.default_rng(9)
    w, x, _, _ = case(rng, n, k, m, 8)
    w[1][:] = rng.integers(0, 255, w[1].shape)
    w[1][:, :] = w[1][:1, :]
    x[1][:, :] = 254 - w[1][:1, :]
    wv, xv = mm.values(*w, 4), mm.values(*x, 8)
    assert_close(run(w, x, 8, n, m, torch.bfloat16), xv @ wv.T, np.abs(xv) @ np.abs(wv).T, torch.bfloat16)
    w[1][:], x[1][:] = 254, 254
    w[0][:], x[0][:] = 2, 0x38
    assert bool(torch.isinf(run(w, x, 8, n, m, torch.float16)).all())
    w[1][:], x[1][:] = 0, 0
    assert bool((run(w, x, 8, n, m, torch.float16) == 0).all())


@pytest.mark.parametrize("bits", [4, 8])
def test_rows_do_not_depend_on_the_batch(bits):
    """A row's result is the same bits in every batch that runs the same kernel."""
    rng = np.random.default_rng(2)
    w, x, _, _ = case(rng, 70, 1056, 16, bits)
    all_rows = run(w, x, bits, 70, 16, torch.float16)
    for i in (0, 7, 15):
        assert torch.equal(run(w, (x[0][i:i + 1], x[1][i:i + 1]), bits, 70, 1, torch.float16), all_rows[i:i + 1])


def test_captured_and_replayed():
    rng = np.random.default_rng(4)
    w, x, _, _ = case(rng, 200, 544, 90, 8)
    wd, xd = mg.to_device(*w, 4), mg.to_device(*x, 8)
    y = torch.zeros((90, 200), dtype=torch.float16, device="cuda")
    few = torch.zeros((9, 200), dtype=torch.float16, device="cuda")
    stream = torch.cuda.Stream()

    def step():
        wq.mx_linear(*wd, *xd, y)
        wq.mx_linear(*wd, xd[0][:9], xd[1][:9], few)

    with torch.cuda.stream(stream):
        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step()
    for seed in range(3):
        c, s = mg.random_matrix(np.random.default_rng(seed), 90, 544, 8, 124, 130)
        nc, ns = mg.to_device(c, s, 8)
        xd[0].view(torch.uint8).copy_(nc.view(torch.uint8))
        xd[1].view(torch.uint8).copy_(ns.view(torch.uint8))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        kept = y.clone(), few.clone()
        step()
        torch.cuda.synchronize()
        assert torch.equal(kept[0], y) and torch.equal(kept[1], few)
