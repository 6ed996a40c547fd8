"""GPU tests of the cache's upkeep at the sizes that it accepts at most."""

from __future__ import annotations

import numpy as np
import pytest

from gpu_util import announce, require_gpu

pytestmark = pytest.mark.gpu


def dev(a):
    import torch

    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, dtype=np.int32))).cuda()


def test_more_pages_wanted_than_32_bits_count():
    """128 rows of 2^24 empty entries want 2^31 pages: the shortfall is reported (up to 2^31 - 1) and nothing changes."""
    import torch

    from paper_2412_15803_amd import wq

    require_gpu()
    width = 1 << 24
    table = torch.full((128, width), -1, dtype=torch.int32, device="cuda")
    for seqs, refs in ((127, [1, 0, 3]), (128, [1, 0, 3]), (128, [2, 1, 1])):
        announce(f"reserve {seqs} x {width} pages, refs {refs}")
        counts, shortfall = dev(refs), dev([-7])
        wq.cache_reserve(table[:seqs], counts, dev([0] * seqs), dev([width] * seqs), 1, shortfall)
        assert shortfall.item() == min(seqs * width - refs.count(0), 2 ** 31 - 1)
        assert counts.tolist() == refs
        assert int(table.max()) == -1
