"""Refusals of the cache's entry points, on the host before any HIP call (no GPU
needed: these calls never reach the device)."""

import ctypes
import os

import pytest

vp = ctypes.c_void_p
A = [0x1000000 * (i + 1) for i in range(12)]  # well aligned, far apart


@pytest.fixture(scope="module")
def L():
    from paper_2412_15803_amd import wq

    if not os.path.exists(wq.LIB_PATH):
        from paper_2412_15803_amd import build

        build.build(verbose=False)
    return wq.lib()


def arrays(*p):
    return (vp * len(p))(*p)


def append(L, k=A[0], v=A[1], kc=A[2], vc=A[3], t=A[4], lens=A[5], starts=A[6], seqs=2, tokens=3, heads=2, dim=64, ks=128, vs=128,
           page=16, pages=8, width=4):
    return L.wq_cache_append(vp(k), vp(v), vp(kc), vp(vc), vp(t), vp(lens), vp(starts), seqs, tokens, heads, dim, ks, vs, page, pages, width, None)


def copy(L, caches=None, n=2, page_bytes=64, pages=8, src=A[4], dst=A[5], count=2):
    return L.wq_cache_copy_pages(arrays(A[0], A[1]) if caches is None else caches, n, page_bytes, pages, vp(src), vp(dst), count, None)


def reserve(L, t=A[0], r=A[1], old=A[2], new=A[3], seqs=2, page=16, pages=8, width=4, short=A[4], ws=A[5], nws=1 << 16):
    return L.wq_cache_reserve(vp(t), vp(r), vp(old), vp(new), seqs, page, pages, width, vp(short), vp(ws), nws, None)


def free(L, t=A[0], r=A[1], lens=A[2], list_=A[3], count=2, window=0, sinks=0, seqs=2, page=16, pages=8, width=4):
    return L.wq_cache_free(vp(t), vp(r), vp(lens), vp(list_), count, window, sinks, seqs, page, pages, width, None)


def fork(L, caches=None, n=1, t=A[1], r=A[2], lens=A[3], src=A[4], dst=A[5], count=2, seqs=4, heads=2, dim=64, page=16, pages=8, width=4,
         short=A[6], ws=A[7], nws=1 << 16):
    return L.wq_cache_fork(arrays(A[0]) if caches is None else caches, n, vp(t), vp(r), vp(lens), vp(src), vp(dst), count, seqs, heads, dim,
                           page, pages, width, vp(short), vp(ws), nws, None)


def compact(L, caches=None, n=1, page_bytes=64, t=A[1], r=A[2], nt=A[3], nr=A[4], live=A[5], seqs=2, pages=8, width=4, ws=A[6], nws=1 << 16):
    return L.wq_cache_compact(arrays(A[0]) if caches is None else caches, n, page_bytes, vp(t), vp(r), vp(nt), vp(nr), vp(live), seqs, pages,
                              width, vp(ws), nws, None)


@pytest.mark.parametrize("call,kwargs,status,needle", [
    (append, dict(k=0), 1, "null"), (append, dict(vc=0), 1, "null"), (append, dict(t=0), 1, "null"), (append, dict(lens=0), 1, "null"),
    (append, dict(seqs=0), 1, "num_seqs"), (append, dict(tokens=0), 1, "num_tokens"), (append, dict(heads=0), 1, "num_kv_heads"),
    (append, dict(heads=257, ks=1 << 20, vs=1 << 20), 1, "num_kv_heads"), (append, dict(dim=12), 2, "head_dim"),
    (append, dict(dim=0), 2, "head_dim"), (append, dict(page=12), 2, "page_size"), (append, dict(page=2048), 2, "page_size"),
    (append, dict(pages=0), 1, "num_pages"), (append, dict(width=0), 1, "max_pages"), (append, dict(starts=0), 1, "q_starts"),
    (append, dict(ks=120), 1, "strides"), (append, dict(vs=132), 1, "strides"), (append, dict(k=A[0] + 8), 3, "aligned"),
    (append, dict(lens=A[5] + 2), 3, "aligned"), (append, dict(vc=A[2] + 64), 1, "overlap"), (append, dict(k=A[2]), 1, "overlap"),
    (copy, dict(n=0), 1, "num_caches"), (copy, dict(n=257), 1, "num_caches"), (copy, dict(caches=arrays(A[0], 0)), 1, "null"),
    (copy, dict(caches=arrays(A[0], A[1] + 8)), 3, "aligned"), (copy, dict(page_bytes=24), 1, "page_bytes"), (copy, dict(page_bytes=0), 1, "page_bytes"),
    (copy, dict(count=9), 1, "count"), (copy, dict(count=-1), 1, "count"), (copy, dict(src=0), 1, "null"), (copy, dict(dst=A[5] + 1), 3, "aligned"),
    (copy, dict(pages=0), 1, "num_pages"),
    (reserve, dict(t=0), 1, "null"), (reserve, dict(short=0), 1, "null"), (reserve, dict(page=3), 2, "page_size"), (reserve, dict(seqs=0), 1, "num_seqs"),
    (reserve, dict(seqs=(1 << 16) + 1), 1, "num_seqs"), (reserve, dict(pages=(1 << 24) + 1), 1, "num_pages"), (reserve, dict(ws=0), 1, "workspace"),
    (reserve, dict(nws=16), 1, "workspace"), (reserve, dict(ws=A[5] + 4), 3, "workspace"), (reserve, dict(r=A[0] + 4), 1, "overlap"),
    (reserve, dict(old=A[0]), 1, "overlap"), (reserve, dict(new=A[3] + 2), 3, "aligned"),
    (free, dict(r=0), 1, "null"), (free, dict(list_=0), 1, "null"), (free, dict(count=3), 1, "count"), (free, dict(window=-1), 1, "window"),
    (free, dict(sinks=(1 << 30) + 1), 1, "sinks"), (free, dict(page=0), 2, "page_size"), (free, dict(r=A[0]), 1, "overlap"),
    (free, dict(list_=A[1]), 1, "overlap"), (free, dict(t=A[0] + 1), 3, "aligned"),
    (fork, dict(lens=0), 1, "null"), (fork, dict(src=0), 1, "null"), (fork, dict(count=5), 1, "count"), (fork, dict(dim=9), 2, "head_dim"),
    (fork, dict(page=24), 2, "page_size"), (fork, dict(ws=0), 1, "workspace"), (fork, dict(src=A[3]), 1, "overlap"), (fork, dict(t=A[0]), 1, "overlap"),
    (fork, dict(caches=arrays(0)), 1, "null"), (fork, dict(short=A[6] + 2), 3, "aligned"),
    (compact, dict(live=0), 1, "null"), (compact, dict(nt=A[1] + 4), 1, "overlap"), (compact, dict(nr=A[1]), 1, "overlap"), (compact, dict(nt=A[0]), 1, "overlap"),
    (compact, dict(page_bytes=8), 1, "page_bytes"), (compact, dict(nws=0), 1, "workspace"), (compact, dict(width=0), 1, "max_pages"),
])
def test_refusals(L, call, kwargs, status, needle):
    assert call(L, **kwargs) == status
    assert needle in L.wq_last_error_message().decode()


def test_nothing_to_do_needs_no_device(L):
    assert copy(L, src=0, dst=0, count=0) == 0
    assert free(L, list_=0, count=0) == 0


def test_workspace_size(L):
    n = ctypes.c_size_t(0)
    assert L.wq_page_workspace_size(1, 1, ctypes.byref(n)) == 0 and n.value > 0
    assert L.wq_page_workspace_size(1 << 24, 1 << 16, ctypes.byref(n)) == 0 and n.value < 1 << 29
    assert L.wq_page_workspace_size(0, 1, ctypes.byref(n)) == 1
    assert L.wq_page_workspace_size(1, 0, ctypes.byref(n)) == 1
    assert L.wq_page_workspace_size(1, 1, None) == 1


def test_binding_refuses_what_is_not_on_the_device():
    import torch

    from paper_2412_15803_amd import wq

    cache = torch.zeros((4, 2, 16, 64), dtype=torch.float16)
    table, lens = torch.zeros((1, 4), dtype=torch.int32), torch.ones(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="device tensor"):
        wq.cache_append(cache[0, :, :1].transpose(0, 1), cache[0, :, :1].transpose(0, 1), cache, cache, table, lens)
    with pytest.raises(ValueError, match="device tensor"):
        wq.cache_set([cache])
    with pytest.raises(ValueError, match="at least one"):
        wq.cache_set([])
    with pytest.raises(TypeError, match="16-bit"):
        wq.cache_set([cache.float()])
