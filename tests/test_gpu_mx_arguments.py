"""Tensors that the binding of the microscaled operators, the norm and the sampler refuses, before anything is queued."""

import pytest
import torch

from gpu_util import require_gpu
from paper_2412_15803_amd import wq

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    require_gpu()


MATRICES = {
    "codes on the host": (lambda c, s: (c.cpu(), s), ValueError, "codes must be a device tensor"),
    "scales on the host": (lambda c, s: (c, s.cpu()), ValueError, "scales must be a device tensor"),
    "short scales": (lambda c, s: (c, s[:, :8]), ValueError, "scales has shape"),
    "turned codes": (lambda c, s: (c.t().contiguous().t(), s), ValueError, "codes must be contiguous"),
    "codes of another type": (lambda c, s: (c.half(), s), TypeError, "codes has dtype"),
    "scales of another type": (lambda c, s: (c, s.float()), TypeError, "scales has dtype"),
    "a row of codes": (lambda c, s: (c[0], s), ValueError, "codes must be 2-D"),
    "a row of scales": (lambda c, s: (c, s[0]), ValueError, "scales must be 2-D"),
    "no codes": (lambda c, s: (None, s), TypeError, "codes must be a torch.Tensor"),
    "a number": (lambda c, s: (c, 3), TypeError, "scales must be a torch.Tensor"),
}


@pytest.mark.parametrize("name", MATRICES)
def test_matrices(name):
    change, error, text = MATRICES[name]
    codes, scales = wq.mx_empty(4, 512, 8)
    x = torch.zeros((4, 512), dtype=torch.float16, device="cuda")
    bad = change(codes, scales)
    for call in (lambda: wq.mx_quantize(x, *bad), lambda: wq.mx_dequantize(*bad, x)):
        with pytest.raises(error, match=text):
            call()


def test_linear():
    w, x = wq.mx_empty(64, 512, 4), wq.mx_empty(40, 512, 8)
    y = torch.zeros((40, 64), dtype=torch.float16, device="cuda")
    for args, error, text in (((x[0], x[1], *x, y), TypeError, "w_codes must be uint8"), ((*w, *wq.mx_empty(40, 544, 8), y), ValueError, "544 columns"),
                              ((*w, *x, y[:39]), ValueError, "y has shape"), ((*w, *x, y.float()), wq.WQError, "dtype"), ((*w, *x, y.t().contiguous().t()), ValueError, "rows of y"),
                              ((*w, *x, y.cpu()), ValueError, "device")):
        with pytest.raises(error, match=text):
            wq.mx_linear(*args)
    for space in (torch.empty(16, dtype=torch.uint8, device="cuda"), torch.empty(1 << 20, dtype=torch.uint8), torch.empty(1 << 20, device="cuda")):
        n, k, m = 64, 4096, 40
        assert wq.mx_linear_workspace_size(n, k, m, 8) > 16
        with pytest.raises((ValueError, wq.WQError), match="workspace"):
            wq.mx_linear(*wq.mx_empty(n, k, 4), *wq.mx_empty(m, k, 8), y, workspace=space)


def test_norm_and_sample():
    x, gain = torch.zeros((4, 512), device="cuda"), torch.zeros(512, device="cuda")
    for args, error, text in ((dict(out=x.half()), TypeError, "out has dtype"), (dict(out=x, residual=x[:3]), ValueError, "residual has shape"), (dict(), wq.WQError, "out or codes"),
                              (dict(codes=wq.mx_empty(4, 512, 8)[0]), ValueError, "go together"), (dict(out=torch.zeros((4, 512))), ValueError, "device")):
        with pytest.raises(error, match=text):
            wq.add_rmsnorm(x, gain, 1e-5, **args)
    with pytest.raises(wq.WQError, match="eps"):
        wq.add_rmsnorm(x, gain, -1.0, out=torch.zeros_like(x))
    random, token = torch.zeros(4, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    for args, error, text in (((x, random[:3], token), ValueError, "random"), ((x, random, token.long()), TypeError, "token"), ((x[0], random, token), ValueError, "logits"),
                              ((x.double(), random, token), TypeError, "logits"), ((x, random.cpu(), token), ValueError, "random")):
        with pytest.raises(error, match=text):
            wq.sample_logits(*args)
    with pytest.raises(wq.WQError, match="workspace"):
        wq.sample_logits(x, random, token, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
