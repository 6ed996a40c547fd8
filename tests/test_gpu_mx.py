"""Microscaled matrices on the GPU: rounding, its inverse, and the gated product,
against NumPy."""

import numpy as np
import pytest
import torch

import mx_gpu as mg
import mx_model as mm
from gpu_util import require_gpu
from paper_2412_15803_amd import wq

pytestmark = pytest.mark.gpu
TYPES = [torch.float16, torch.bfloat16, torch.float32]


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    require_gpu()


def values_of(t):
    return t.float().cpu().numpy().astype(np.float64)


def hard_rows(rng, cols, dtype):
    """Rows with what rounding can go wrong at: ties, borders of the scale, zeros of
    both signs, denormals, the type's largest value, NaN and infinities."""
    info = torch.finfo(dtype)
    rows = []
    for bits in (4, 8):
        g = mm.grid(bits)
        ties = (g[1:] + g[:-1]) / 2
        for e in (-6, 0, 5):
            v = np.resize(np.concatenate([ties, -ties]), cols)
            v.reshape(-1, 32)[:, 7] = g[-1]  # the block's largest, so that the scale is 2^e
            rows.append(v * 2.0 ** e)
        top = np.full(cols, 0.5)
        top[0::32] = g[-1]
        rows += [top, -top, np.nextafter(np.float32(g[-1]), np.float32(1e9)).astype(np.float64) * np.ones(cols)]
    rows.append(np.zeros(cols))
    rows.append(-np.zeros(cols))
    rows.append(np.where(np.arange(cols) % 2, info.max, -info.max / 3))
    rows.append(rng.standard_normal(cols) * info.tiny / 4)
    rows.append(np.where(np.arange(cols) % 5 == 0, info.tiny * info.eps, 0.0))
    for bad in (np.nan, np.inf, -np.inf):
        v = rng.standard_normal(cols)
        v[::64] = bad
        rows.append(v)
    return np.stack(rows)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("rows,cols,stride", [(1, 32, 32), (3, 64, 72), (1, 4096, 4096), (77, 2080, 2080), (5, 544, 1000), (1030, 96, 96), (2, 20000 * 32, 20000 * 32)])
def test_quantize(dtype, bits, rows, cols, stride):
    rng = np.random.default_rng(rows * cols + bits)
    wide = torch.full((rows, stride), float("nan"), dtype=dtype, device="cuda")
    x = wide[:, :cols]
    x.copy_(torch.from_numpy(rng.standard_normal((rows, cols)) * 2.0 ** rng.integers(-8, 8, (rows, 1))))
    codes, scales = mg.room(rows, cols, bits)
    wq.mx_quantize(x, codes, scales)
    got, s, padding = mg.to_host(codes, scales, bits)
    want, want_s = mm.quantize(values_of(x), bits)
    assert np.array_equal(s, want_s)
    assert np.array_equal(got, want)
    assert np.all(padding == 0xA5)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("cols", [32, 288])
def test_quantize_hard_values(dtype, bits, cols):
    x = torch.from_numpy(hard_rows(np.random.default_rng(bits), cols, dtype)).to(dtype).cuda()
    codes, scales = mg.room(*x.shape, bits)
    wq.mx_quantize(x, codes, scales)
    got, s, _ = mg.to_host(codes, scales, bits)
    want, want_s = mm.quantize(values_of(x), bits)
    assert np.array_equal(s, want_s)
    assert np.array_equal(got, want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("rows,cols,stride", [(1, 32, 64), (3, 2080, 4160), (9, 544, 1200), (300, 1024, 2048)])
def test_quantize_gated(dtype, bits, rows, cols, stride):
    """silu in fp32: exp's argument is rounded (|g| <= 16: relative 2^-20 of exp), then five operations of 2^-23 at
    most each: below 2^-19 in all."""
    rng = np.random.default_rng(rows + cols)
    x = torch.zeros((rows, stride), dtype=dtype, device="cuda")[:, :2 * cols]
    x.copy_(torch.from_numpy(np.clip(rng.standard_normal((rows, 2 * cols)) * 3, -16, 16)))
    codes, scales = mg.room(rows, cols, bits)
    wq.mx_quantize(x, codes, scales, gated=True)
    v = values_of(x)
    g, u = v[:, :cols], v[:, cols:]
    got, s, padding = mg.to_host(codes, scales, bits)
    mm.check_rounded(got, s, g / (1 + np.exp(-g)) * u, bits, 2.0 ** -19)
    assert np.all(padding == 0xA5)


def test_gated_far_from_zero():
    """Gates whose exponential overflows or vanishes, and values that are none."""
    x = torch.zeros((4, 64), device="cuda")
    x[0, :32], x[0, 32:] = -200.0, 3.0
    x[1, :32], x[1, 32:] = 200.0, 0.5
    x[2, :32], x[2, 32:], x[2, 5] = 1.0, 1.0, float("nan")
    x[3, :32], x[3, 32:], x[3, 37] = 1.0, 1.0, float("inf")
    codes, scales = mg.room(4, 32, 8)
    wq.mx_quantize(x, codes, scales, gated=True)
    got, s, _ = mg.to_host(codes, scales, 8)
    assert np.all(mm.values(got, s, 8)[0] == 0)
    assert np.all(np.abs(mm.values(got, s, 8)[1] - 100) <= 100 * 2.0 ** -4)
    assert s[2, 0] == 255 and s[3, 0] == 255 and np.all(got[2:] == 0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("rows,cols,stride", [(1, 32, 32), (256, 64, 72), (77, 2080, 2080)])
def test_dequantize(dtype, bits, rows, cols, stride):
    rng = np.random.default_rng(rows)
    codes, scales = mg.random_matrix(rng, rows, cols, bits, 0, 255)
    if bits == 8:
        codes[0, :] = np.resize(np.arange(256), cols)  # NaN codes among them
        scales[0] = 127
    wide = torch.full((rows, stride), 7.0, dtype=dtype, device="cuda")
    wq.mx_dequantize(*mg.to_device(codes, scales, bits), wide[:, :cols])
    want = torch.from_numpy(mm.values(codes, scales, bits))
    # Rounded once: through fp32, which holds every product exactly or as infinity.
    want = want.float().to(dtype)
    got = wide[:, :cols].cpu()
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    assert bool(same.all())
    assert bool((wide[:, cols:] == 7.0).all())


@pytest.mark.parametrize("bits", [4, 8])
def test_there_and_back_is_the_same(bits):
    """Values that a matrix can hold come back as they are, and as the same codes."""
    rng = np.random.default_rng(3)
    codes, scales = mg.random_matrix(rng, 64, 256, bits, 110, 140)
    codes[:, ::32] = len(mm.grid(bits)) - 1  # the largest value, so that the scale is determined
    out = torch.empty((64, 256), device="cuda")
    wq.mx_dequantize(*mg.to_device(codes, scales, bits), out)
    c, s = mg.room(64, 256, bits)
    wq.mx_quantize(out, c, s)
    got, got_s, _ = mg.to_host(c, s, bits)
    assert np.array_equal(got, codes) and np.array_equal(got_s, scales)


def test_captured_and_replayed():
    x = torch.zeros((33, 1088), dtype=torch.bfloat16, device="cuda")
    codes, scales = mg.room(33, 544, 8)
    out = torch.empty((33, 544), device="cuda")

    def step():
        wq.mx_quantize(x, codes, scales, gated=True)
        wq.mx_dequantize(codes, scales, out)

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in range(3):
        x.copy_(torch.randn(x.shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        replayed = out.clone()
        step()
        assert torch.equal(replayed, out)
