"""paged_attention without a workspace, queued on a stream that is not the current one."""

from __future__ import annotations

import pytest

from gpu_util import require_gpu

pytestmark = pytest.mark.gpu


def test_the_workspace_belongs_to_the_stream_of_the_call(monkeypatch):
    import torch

    from paper_2412_15803_amd import wq

    require_gpu()
    g = torch.Generator(device="cuda").manual_seed(3)
    pages, hkv, page, d, n = 400, 2, 16, 128, 6000
    k, v = (torch.randn((pages, hkv, page, d), generator=g, device="cuda").half() for _ in range(2))
    q = torch.randn((1, 8, d), generator=g, device="cuda").half()
    table = torch.randperm(pages, generator=g, device="cuda").int()[None, :375].contiguous()
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    want, out = torch.empty_like(q), torch.empty_like(q)
    wq.paged_attention(q, k, v, table, lens, want, d ** -0.5, n, workspace=wq.paged_workspace(q, n, hkv))
    made, make = [], wq.paged_workspace

    def recorded(*args):
        made.append(torch.cuda.current_stream().cuda_stream)
        return make(*args)

    monkeypatch.setattr(wq, "paged_workspace", recorded)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    wq.paged_attention(q, k, v, table, lens, out, d ** -0.5, n, stream=side)
    wq.paged_attention(q, k, v, table, lens, torch.empty_like(q), d ** -0.5, n)
    torch.cuda.synchronize()
    assert made == [side.cuda_stream, torch.cuda.current_stream().cuda_stream]
    assert torch.equal(out, want)
