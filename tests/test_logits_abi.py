"""Refusals of wq_process_logits, on the host before any HIP call (no GPU needed:
these calls never reach the device)."""

import ctypes
import os

import pytest

A = [0x1000000 * (i + 1) for i in range(16)]  # well aligned, far apart
GOOD = dict(logits=A[0], out=A[1], token=A[2], mask=A[3], history=A[4], history_lens=A[5], prompt_lens=A[6], repetition=A[7], frequency=A[8],
            presence=A[9], bias_ids=A[10], bias_values=A[11], bias_lens=A[12], rows=2, vocab=100, logits_stride=100, out_stride=104, mask_stride=4,
            history_size=10, bias_size=3, dtype=0)


@pytest.fixture(scope="module")
def wq():
    from paper_2412_15803_amd import wq as module

    if not os.path.exists(module.LIB_PATH):
        from paper_2412_15803_amd import build

        build.build(verbose=False)
    module.lib()
    return module


@pytest.mark.parametrize("change,status,needle", [
    (dict(logits=None), 1, "null"), (dict(out=None), 1, "null"), (dict(rows=0), 1, "rows"), (dict(rows=65536), 1, "rows"), (dict(vocab=0), 1, "vocab"),
    (dict(vocab=(1 << 24) + 1), 1, "vocab"), (dict(dtype=3), 2, "dtype"), (dict(dtype=-1), 2, "dtype"), (dict(logits_stride=99), 1, "logits_stride"),
    (dict(out_stride=99), 1, "out_stride"), (dict(mask_stride=3), 1, "mask_stride"), (dict(history_size=0), 1, "history_size"),
    (dict(history=None), 1, "history"), (dict(bias_ids=None), 1, "bias_ids"), (dict(bias_values=None), 1, "bias_values"), (dict(bias_size=0), 1, "bias_size"),
    (dict(logits=A[0] + 1), 3, "aligned"), (dict(logits=A[0] + 2, dtype=2), 3, "aligned"), (dict(token=A[2] + 2), 3, "aligned"), (dict(bias_lens=A[12] + 1), 3, "aligned"),
    (dict(out=A[0]), 1, "overlap"), (dict(out=A[0] + 64), 1, "overlap"), (dict(token=A[0]), 1, "overlap"), (dict(mask=A[1]), 1, "overlap"),
    (dict(history_lens=A[2]), 1, "overlap"),
])
def test_refusals(wq, change, status, needle):
    call = wq.WqLogitsCall(**{**GOOD, **change})
    L = wq.lib()
    assert L.wq_process_logits(ctypes.addressof(call), None, 0, None) == status
    assert needle in L.wq_last_error_message().decode()


def test_workspace_is_checked(wq):
    L, n = wq.lib(), ctypes.c_size_t(0)
    big = wq.WqLogitsCall(**{**GOOD, "vocab": 100000, "logits_stride": 100000, "out_stride": 100000, "mask_stride": 3125})
    assert L.wq_process_logits_workspace_size(2, 100000, 0, ctypes.byref(n)) == 0 and n.value > 0
    for pointer, size, status in ((None, 0, 1), (A[13], n.value - 1, 1), (A[13] + 8, n.value, 3), (A[1], n.value, 1)):
        assert L.wq_process_logits(ctypes.addressof(big), pointer, size, None) == status
        assert "workspace" in L.wq_last_error_message().decode()
    assert L.wq_process_logits_workspace_size(2, 100, 2, ctypes.byref(n)) == 0 and n.value == 0
    assert L.wq_process_logits_workspace_size(0, 100, 2, ctypes.byref(n)) == 1
    assert L.wq_process_logits_workspace_size(2, 100, 9, ctypes.byref(n)) == 2
    assert L.wq_process_logits_workspace_size(2, 100, 0, None) == 1
    assert L.wq_process_logits(None, None, 0, None) == 1


def test_binding_refuses_before_the_library(wq):
    import torch

    x = torch.zeros((2, 8))
    with pytest.raises(ValueError, match="device tensor"):
        wq.process_logits(x, x)
    with pytest.raises(TypeError, match="share"):
        wq.process_logits(x, x.half())
    with pytest.raises(ValueError, match=r"\[R, V\]"):
        wq.process_logits(x[0], x[0])
