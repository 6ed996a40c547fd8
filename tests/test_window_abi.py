"""Refusals of wq_window_attention, on the host before any HIP call (no GPU
needed: these calls never reach the device)."""

import ctypes
import math
import os

import pytest

A = [0x100000000 * (i + 1) for i in range(10)]  # well aligned, far apart
vp = ctypes.c_void_p


@pytest.fixture(scope="module")
def L():
    from paper_2412_15803_amd import wq

    if not os.path.exists(wq.LIB_PATH):
        from paper_2412_15803_amd import build

        build.build(verbose=False)
    return wq.lib()


def call(L, q=A[0], k=A[1], v=A[2], t=A[3], lens=A[4], starts=A[5], out=A[6], seqs=2, tokens=6, most=4, hq=8, hkv=2, dim=64, qs=512, os_=512,
         page=16, pages=10, width=4, max_len=64, window=32, sinks=4, scale=0.125, dtype=0, ws=A[7], nws=1 << 30):
    return L.wq_window_attention(vp(q), vp(k), vp(v), vp(t), vp(lens), vp(starts), vp(out), seqs, tokens, most, hq, hkv, dim, qs, os_, page,
                                 pages, width, max_len, window, sinks, scale, dtype, vp(ws), nws, None)


@pytest.mark.parametrize("kwargs,status,needle", [
    (dict(q=0), 1, "null"), (dict(k=0), 1, "null"), (dict(v=0), 1, "null"), (dict(t=0), 1, "null"), (dict(lens=0), 1, "null"), (dict(out=0), 1, "null"),
    (dict(seqs=0), 1, "num_seqs"), (dict(seqs=1 << 17), 1, "num_seqs"), (dict(tokens=0), 1, "num_tokens"), (dict(most=0), 1, "max_query_len"),
    (dict(most=7), 1, "max_query_len"), (dict(hkv=0), 1, "num_kv_heads"), (dict(hkv=257, hq=257), 1, "num_kv_heads"), (dict(hq=7), 1, "multiple"),
    (dict(hq=0), 1, "multiple"), (dict(hq=34), 2, "query heads"), (dict(dim=96), 2, "head_dim"), (dict(dim=256), 2, "head_dim"),
    (dict(max_len=0), 1, "max_seq_len"), (dict(max_len=1 << 25), 1, "max_seq_len"), (dict(window=-1), 1, "window"), (dict(sinks=-1), 1, "sinks"),
    (dict(window=(1 << 30) + 1), 1, "window"), (dict(page=0), 2, "page_size"), (dict(page=48), 2, "page_size"), (dict(page=2048), 2, "page_size"),
    (dict(dtype=2), 2, "dtype"), (dict(dtype=-1), 2, "dtype"), (dict(pages=0), 1, "num_pages"), (dict(width=0), 1, "max_pages"),
    (dict(starts=0), 1, "q_starts"), (dict(starts=0, seqs=6), 1, "q_starts"), (dict(qs=504), 1, "strides"), (dict(os_=516), 1, "strides"),
    (dict(scale=math.inf), 1, "finite"), (dict(scale=math.nan), 1, "finite"), (dict(q=A[0] + 8), 3, "aligned"), (dict(out=A[6] + 2), 3, "aligned"),
    (dict(v=A[2] + 8), 3, "aligned"), (dict(lens=A[4] + 2), 3, "aligned"), (dict(starts=A[5] + 1), 3, "aligned"), (dict(out=A[0]), 1, "overlap"),
    (dict(out=A[1] + 64), 1, "overlap"), (dict(out=A[3]), 1, "overlap"),
])
def test_refusals(L, kwargs, status, needle):
    assert call(L, **kwargs) == status
    assert needle in L.wq_last_error_message().decode()


def test_workspace_is_checked(L):
    n = ctypes.c_size_t(0)
    sizes = (1, 1, 1, 8, 2, 64, 4096, 4096, 0)
    assert L.wq_window_attention_workspace_size(*sizes, ctypes.byref(n)) == 0 and n.value > 0
    split = dict(starts=0, seqs=1, tokens=1, most=1, max_len=4096, width=256, window=4096, sinks=0)
    for ws, nws, status in ((0, 0, 1), (A[7], n.value - 1, 1), (A[7] + 8, n.value, 3), (A[6], n.value, 1), (A[1], n.value, 1)):
        assert call(L, ws=ws, nws=nws, **split) == status
        assert "workspace" in L.wq_last_error_message().decode()
    assert L.wq_window_attention_workspace_size(*sizes, None) == 1
    assert L.wq_window_attention_workspace_size(1, 1, 1, 8, 2, 80, 4096, 4096, 0, ctypes.byref(n)) == 2
    # Long batches of one-token sequences and long prompts need little or none.
    assert L.wq_window_attention_workspace_size(1024, 1024, 1, 32, 8, 128, 1 << 20, 4096, 4, ctypes.byref(n)) == 0 and n.value == 0
    assert L.wq_window_attention_workspace_size(1, 8192, 8192, 32, 8, 128, 8192, 4096, 4, ctypes.byref(n)) == 0 and n.value == 0


def test_workspace_stays_bounded(L):
    n = ctypes.c_size_t(0)
    for seqs in (1, 3, 17, 100, 1000, 1 << 16):
        for most in (1, 2, 16, 500, 4096):
            for heads in ((1, 1), (24, 8), (32, 8), (16, 1), (256, 256)):
                for length in (1, 700, 1 << 15, 1 << 24):
                    if seqs * most <= 1 << 22 and seqs * most * heads[0] < 1 << 30:
                        assert L.wq_window_attention_workspace_size(seqs, seqs * most, most, *heads, 128, length, length, 4, ctypes.byref(n)) == 0
                        assert n.value < 1 << 30, (seqs, most, heads, length)


def test_binding_refuses_before_the_library():
    import torch

    from paper_2412_15803_amd import wq

    q, cache = torch.zeros((1, 4, 64)).half(), torch.zeros((3, 2, 16, 64)).half()
    table, lens = torch.zeros((1, 3), dtype=torch.int32), torch.ones(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="device tensor"):
        wq.window_attention(q, cache, cache, table, lens, q, 1.0, 16, 8)
    with pytest.raises(ValueError, match="head_dim"):
        wq.window_attention(q[:, :, :32], cache, cache, table, lens, q, 1.0, 16, 8)
    with pytest.raises(TypeError, match="16-bit"):
        wq.window_attention(q, cache.float(), cache, table, lens, q, 1.0, 16, 8)
    with pytest.raises(TypeError, match="fp16 or bf16"):
        wq.window_attention(q, cache.view(torch.int16), cache, table, lens, q, 1.0, 16, 8)
