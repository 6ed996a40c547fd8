"""Refusals of the microscaled operators, the norm and the sampler, on the host before any
HIP call (no GPU needed: these calls never reach the device)."""

import ctypes
import os

import pytest

A = [0x100000000 * (i + 1) for i in range(16)]  # well aligned, far apart


@pytest.fixture(scope="module")
def wq():
    from paper_2412_15803_amd import wq as module

    if not os.path.exists(module.LIB_PATH):
        from paper_2412_15803_amd import build

        build.build(verbose=False)
    module.lib()
    return module


def refused(wq, status, needle, got):
    assert got == status
    assert needle in wq.last_error_message()


QUANTIZE = dict(x=A[0], codes=A[1], scales=A[2], rows=4, cols=64, x_stride=64, dtype=0, gated=0, format=8)


@pytest.mark.parametrize("change,status,needle", [
    (dict(x=None), 1, "null"), (dict(codes=None), 1, "null"), (dict(scales=None), 1, "null"), (dict(rows=0), 1, "rows"), (dict(rows=(1 << 24) + 1), 1, "rows"),
    (dict(cols=0), 1, "cols"), (dict(cols=48), 2, "multiple of 32"), (dict(cols=(1 << 20) + 32), 1, "cols"), (dict(dtype=3), 2, "dtype"), (dict(gated=2), 1, "gated"),
    (dict(format=5), 2, "format"), (dict(x_stride=56), 1, "x_stride"), (dict(x_stride=68), 1, "x_stride"), (dict(gated=1, x_stride=120), 1, "x_stride"),
    (dict(x=A[0] + 8), 3, "x must be"), (dict(codes=A[1] + 8), 3, "codes"), (dict(scales=A[2] + 4), 3, "scales"), (dict(codes=A[0] + 16), 1, "overlap"),
    (dict(scales=A[1]), 1, "overlap"), (dict(scales=A[0] + 496), 1, "overlap"),
])
def test_quantize(wq, change, status, needle):
    refused(wq, status, needle, wq.lib().wq_mx_quantize(*{**QUANTIZE, **change}.values(), None))


DEQUANTIZE = dict(codes=A[0], scales=A[1], out=A[2], rows=4, cols=64, out_stride=64, format=4, dtype=2)


@pytest.mark.parametrize("change,status,needle", [
    (dict(out=None), 1, "null"), (dict(codes=None), 1, "null"), (dict(scales=None), 1, "null"), (dict(rows=-1), 1, "rows"), (dict(cols=33), 2, "multiple of 32"),
    (dict(out_stride=63), 1, "out_stride"), (dict(format=0), 2, "format"), (dict(dtype=-1), 2, "dtype"), (dict(out=A[2] + 4), 3, "out must be"),
    (dict(codes=A[0] + 1), 3, "codes"), (dict(out=A[0]), 1, "overlap"), (dict(out=A[1] - 16), 1, "overlap"),
])
def test_dequantize(wq, change, status, needle):
    refused(wq, status, needle, wq.lib().wq_mx_dequantize(*{**DEQUANTIZE, **change}.values(), None))


LINEAR = dict(w_codes=A[0], w_scales=A[1], x_codes=A[2], x_scales=A[3], y=A[4], n=100, k=1024, m=70, y_stride=100, x_format=8, dtype=0, workspace=A[5], bytes=1 << 31)


@pytest.mark.parametrize("change,status,needle", [
    (dict(w_codes=None), 1, "null"), (dict(w_scales=None), 1, "null"), (dict(x_codes=None), 1, "null"), (dict(x_scales=None), 1, "null"), (dict(y=None), 1, "null"),
    (dict(n=0), 1, "N"), (dict(k=0), 1, "K"), (dict(k=1000), 2, "K must be"), (dict(k=1 << 21), 1, "K"), (dict(m=0), 1, "M"), (dict(m=(1 << 24) + 1), 1, "M"),
    (dict(x_format=3), 2, "x_format"), (dict(dtype=2), 2, "dtype"), (dict(y_stride=99), 1, "y_stride"), (dict(w_codes=A[0] + 8), 3, "aligned"),
    (dict(x_scales=A[3] + 1), 3, "aligned"), (dict(y=A[4] + 1), 3, "aligned"), (dict(y=A[0]), 1, "overlap"), (dict(y=A[3] + 16), 1, "overlap"),
    (dict(y=A[2] - 2), 1, "overlap"),
])
def test_linear(wq, change, status, needle):
    refused(wq, status, needle, wq.lib().wq_mx_linear(*{**LINEAR, **change}.values(), None))


def test_linear_workspace(wq):
    L, n = wq.lib(), ctypes.c_size_t(0)
    for sizes, status in (((0, 32, 1, 8), 1), ((1, 33, 1, 8), 2), ((1, 32, 0, 8), 1), ((1, 32, 1, 6), 2)):
        assert L.wq_mx_linear_workspace_size(*sizes, ctypes.byref(n)) == status
    assert L.wq_mx_linear_workspace_size(1, 32, 1, 8, None) == 1
    for bits in (4, 8):
        for n_, k, m in ((1, 32, 1), (4096, 14336, 33), (28672, 4096, 8192), (4096, 4096, 200), (64, 1 << 20, 300)):
            assert L.wq_mx_linear_workspace_size(n_, k, m, bits, ctypes.byref(n)) == 0
            need = n.value
            assert need % 16 == 0
            if need:
                call = {**LINEAR, **dict(n=n_, k=k, m=m, y_stride=n_, x_format=bits)}
                for pointer, size, status in ((None, 0, 1), (A[5], need - 1, 1), (A[5] + 8, need, 3), (A[4], need, 1), (A[0], need, 1)):
                    refused(wq, status, "workspace", L.wq_mx_linear(*{**call, "workspace": pointer, "bytes": size}.values(), None))


NORM = dict(x=A[0], residual=A[1], weight=A[2], total=A[3], out=A[4], codes=A[5], scales=A[6], rows=4, dim=64, x_stride=64, residual_stride=72, total_stride=64,
            out_stride=64, dtype=0, format=8, eps=1e-5)


@pytest.mark.parametrize("change,status,needle", [
    (dict(x=None), 1, "null"), (dict(weight=None), 1, "null"), (dict(out=None, codes=None, scales=None), 1, "out or codes"), (dict(codes=None), 1, "go together"),
    (dict(scales=None), 1, "go together"), (dict(rows=0), 1, "rows"), (dict(rows=(1 << 21) + 1), 1, "rows"), (dict(dim=0), 1, "dim"), (dict(dim=40), 2, "multiple of 32"),
    (dict(dim=32800), 1, "dim"), (dict(dtype=4), 2, "dtype"), (dict(format=7), 2, "format"), (dict(eps=-1.0), 1, "eps"), (dict(eps=float("nan")), 1, "eps"),
    (dict(eps=float("inf")), 1, "eps"), (dict(x_stride=63), 1, "stride of x"), (dict(residual_stride=68), 1, "stride of residual"), (dict(total_stride=0), 1, "stride of total"),
    (dict(out_stride=1 << 33), 1, "stride of out"), (dict(x=A[0] + 2), 3, "aligned"), (dict(weight=A[2] + 8), 3, "aligned"), (dict(scales=A[6] + 8), 3, "aligned"),
    (dict(out=A[3]), 1, "outputs overlap"), (dict(codes=A[4] + 16), 1, "overlap"), (dict(total=A[2]), 1, "weight"), (dict(out=A[0] + 16), 1, "input"),
    (dict(total=A[1]), 1, "input"), (dict(codes=A[0]), 1, "input"), (dict(total=A[0], residual=A[0] + 16), 1, "input"),
])
def test_norm(wq, change, status, needle):
    call = wq.WqNormCall(**{**NORM, **change})
    refused(wq, status, needle, wq.lib().wq_add_rmsnorm(ctypes.addressof(call), None))


SAMPLE = dict(logits=A[0], random=A[1], temperature=A[2], top_k=A[3], top_p=A[4], min_p=A[5], token=A[6], share=A[7], rows=3, vocab=1000, logits_stride=1003, dtype=2)


@pytest.mark.parametrize("change,status,needle", [
    (dict(logits=None), 1, "null"), (dict(random=None), 1, "null"), (dict(token=None), 1, "null"), (dict(rows=0), 1, "rows"), (dict(rows=65536), 1, "rows"),
    (dict(vocab=0), 1, "vocab"), (dict(vocab=(1 << 20) + 1), 1, "vocab"), (dict(dtype=3), 2, "dtype"), (dict(logits_stride=999), 1, "logits_stride"),
    (dict(logits=A[0] + 2), 3, "aligned"), (dict(random=A[1] + 2), 3, "aligned"), (dict(token=A[6] + 1), 3, "aligned"), (dict(share=A[7] + 2), 3, "aligned"),
    (dict(top_k=A[3] + 1), 3, "aligned"), (dict(token=A[0] + 400), 1, "overlap"), (dict(share=A[6] + 8), 1, "overlap"), (dict(token=A[1]), 1, "overlap"),
    (dict(share=A[5] + 4), 1, "overlap"),
])
def test_sample(wq, change, status, needle):
    call = wq.WqSampleCall(**{**SAMPLE, **change})
    refused(wq, status, needle, wq.lib().wq_sample_logits(ctypes.addressof(call), A[8], 1 << 31, None))


def test_sample_workspace(wq):
    L, n = wq.lib(), ctypes.c_size_t(0)
    assert L.wq_sample_logits(None, None, 0, None) == 1
    for sizes, status in (((0, 5, 0), 1), ((1, 0, 0), 1), ((1, 5, 7), 2)):
        assert L.wq_sample_logits_workspace_size(*sizes, ctypes.byref(n)) == status
    assert L.wq_sample_logits_workspace_size(1, 5, 0, None) == 1
    for rows, vocab in ((1, 10), (1, 128256), (48, 128256), (65535, 1 << 20), (256, 100277)):
        assert L.wq_sample_logits_workspace_size(rows, vocab, 0, ctypes.byref(n)) == 0
        need = n.value
        assert need % 16 == 0
        if need:
            call = wq.WqSampleCall(**{**SAMPLE, **dict(rows=rows, vocab=vocab, logits_stride=vocab, dtype=0)})
            for pointer, size, status in ((None, 0, 1), (A[8], need - 1, 1), (A[8] + 8, need, 3), (A[6], need, 1), (A[1], need, 1)):
                refused(wq, status, "workspace", L.wq_sample_logits(ctypes.addressof(call), pointer, size, None))


def test_binding_refuses_before_the_library(wq):
    import torch

    x = torch.zeros((2, 64))
    codes, scales = wq.mx_empty(2, 64, 8, device="cpu")
    assert codes.dtype == torch.float8_e4m3fn and codes.shape == (2, 64) and scales.shape == (2, 16)
    assert wq.mx_empty(2, 544, 4, device="cpu")[0].shape == (2, 272) and wq.mx_scale_stride(544) == 32
    for bits, cols in ((6, 64), (8, 40)):
        with pytest.raises(ValueError):
            wq.mx_empty(2, cols, bits, device="cpu")
    for call in (lambda: wq.mx_quantize(x, codes, scales), lambda: wq.mx_dequantize(codes, scales, x), lambda: wq.mx_linear(codes, scales, codes, scales, x.half()),
                 lambda: wq.add_rmsnorm(x, x[0], 1e-5, out=x), lambda: wq.sample_logits(x, x[0, :2], torch.zeros(2, dtype=torch.int32))):
        with pytest.raises(ValueError, match="device tensor"):
            call()
    with pytest.raises(TypeError, match="x must be"):
        wq.mx_quantize(x.int(), codes, scales)
    with pytest.raises(ValueError, match="2-D"):
        wq.mx_quantize(x, codes[0], scales)
    with pytest.raises(ValueError, match=r"\[R, D\]"):
        wq.add_rmsnorm(x[0], x[0], 1e-5, out=x[0])
    with pytest.raises(ValueError, match=r"\[R, V\]"):
        wq.sample_logits(x[0], x[0], x[0])


def test_packed_calls(wq):
    """The bytes that the binding passes are those of the structures."""
    pointers, sizes = list(range(1, 9)), [1 << (4 * i) for i in range(8)]
    assert wq._NORM_CALL(*pointers[:7], *sizes, 0.5) == bytes(wq.WqNormCall(*pointers[:7], *sizes, 0.5))
    assert wq._SAMPLE_CALL(*pointers, *sizes[:4]) == bytes(wq.WqSampleCall(*pointers, *sizes[:4]))
