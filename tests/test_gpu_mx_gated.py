"""The gated product over the range of its gates, against float64 and the bound of include/wq_mx.h.

Rounded codes hide an error of the product but where it lies next to a border between two of them, so there are
many values, and a block's are of one size: none is hidden by the scale of a larger one."""

import numpy as np
import pytest
import torch

import mx_gpu as mg
import mx_model as mm
from gpu_util import require_gpu
from paper_2412_15803_amd import wq

pytestmark = pytest.mark.gpu
REL = 2.0 ** -20  # the header's; what it adds, 2^-148 (1 + |up|), is below a 2^-20th of this for every value here


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    require_gpu()


def check(gate, up, dtype, bits):
    x = torch.from_numpy(np.concatenate([gate, up], axis=1)).to(dtype).cuda()
    rows, cols = gate.shape
    codes, scales = mg.room(rows, cols, bits)
    wq.mx_quantize(x, codes, scales, gated=True)
    v = x.double().cpu().numpy()
    g, u = v[:, :cols], v[:, cols:]
    e = np.exp(-np.abs(g))
    silu = g * np.where(g < 0, e, 1.0) / (1 + e)
    c, s, _ = mg.to_host(codes, scales, bits)
    mm.check_rounded(c, s, silu * u, bits, REL)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("low,high", [(-87, -60), (-60, -30), (-30, -10), (-10, -2), (-2, 0), (0, 2), (2, 20), (20, 90)])
def test_gates(dtype, bits, low, high):
    rng = np.random.default_rng(high + 100)
    cols, rows = 1024, 512
    centre = rng.uniform(low + 0.5, high - 0.5, (rows, cols // 32, 1))
    gate = np.clip(centre + rng.uniform(-0.5, 0.5, (rows, cols // 32, 32)), low, high).reshape(rows, cols)
    up = rng.uniform(0.5, 2.0, (rows, cols)) * rng.choice([-1.0, 1.0], (rows, cols))
    check(gate, up, dtype, bits)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_gates_and_factors_of_any_size(dtype):
    """Gates whose exponential vanishes, up to the type's largest, and small ones; factors that bring the product back."""
    rng = np.random.default_rng(4)
    sizes = np.array([1e-30, 1e-10, 1e-3, 88.0, 130.0, 1e4, 1e10, 1e30, 1e38, 3.3e38])[:, None]
    gate = sizes * rng.uniform(0.97, 1.0, (len(sizes), 320))
    up = rng.uniform(0.5, 2.0, gate.shape) / np.maximum(sizes, 1)
    check(gate, up, dtype, 8)
    check(-gate[:3], up[:3], dtype, 8)
    # Far below 0: silu's exact value times the factor is below 2^-120, and what comes out no larger.
    far = torch.from_numpy(np.concatenate([-gate[3:], up[3:]], axis=1)).to(dtype).cuda()
    codes, scales = mg.room(len(far), 320, 8)
    wq.mx_quantize(far, codes, scales, gated=True)
    c, s, _ = mg.to_host(codes, scales, 8)
    assert np.all(np.abs(mm.values(c, s, 8)) <= 2.0 ** -120)
