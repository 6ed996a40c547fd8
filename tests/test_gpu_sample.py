"""The choice of a word by chance on the GPU against the model in float64."""

import math

import numpy as np
import pytest
import torch

import sample_model as sm
from gpu_util import require_gpu
from paper_2412_15803_amd import wq

pytestmark = pytest.mark.gpu
TYPES = [torch.float16, torch.bfloat16, torch.float32]
OPTIONS = [dict(), dict(temperature=0.7), dict(top_k=1), dict(top_k=7, temperature=1.3), dict(top_k=300), dict(top_p=0.9), dict(top_p=0.3, temperature=2.0),
           dict(min_p=0.05), dict(top_k=40, top_p=0.95, temperature=0.8), dict(top_k=1000, top_p=0.5, min_p=0.1), dict(top_p=0.999, min_p=0.001), dict(temperature=0.0)]


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    require_gpu()


def column(options, name, default, dtype):
    if all(name not in o for o in options):
        return None
    return torch.tensor([o.get(name, default) for o in options], dtype=dtype, device="cuda")


def call(logits, random, options, **more):
    rows = logits.shape[0]
    token = torch.full((rows,), -7, dtype=torch.int32, device="cuda")
    share = torch.full((rows,), -7.0, device="cuda")
    wq.sample_logits(logits, torch.tensor(random, dtype=torch.float32, device="cuda"), token, temperature=column(options, "temperature", 1.0, torch.float32),
                     top_k=column(options, "top_k", 0, torch.int32), top_p=column(options, "top_p", 1.0, torch.float32),
                     min_p=column(options, "min_p", 0.0, torch.float32), share=share, **more)
    return token.cpu().tolist(), share.cpu().tolist()


def fp32(option):
    """The parameters as the device has them: fp32 values, exactly."""
    return {k: float(np.float32(v)) if k != "top_k" else v for k, v in option.items()}


def compare(logits, options, rng, tries=3):
    """Random numbers clear of the borders, so that an exact implementation has one answer."""
    x = logits.double().cpu().numpy()
    weights = [sm.stays(list(row), **fp32(o)) for row, o in zip(x, options)]
    for _ in range(tries):
        random = []
        for w in weights:
            u = float(np.float32(rng.random()))
            while w is not None and not sm.clear_of_borders(w, u):
                u = float(np.float32(rng.random()))
            random.append(min(u, 1 - 2.0 ** -24))
        token, share = call(logits, random, options)
        for i, w in enumerate(weights):
            want, part = sm.choose(w, random[i])
            assert token[i] == want, (i, options[i], random[i], token[i], want)
            assert abs(share[i] - part) <= 2.0 ** -23 * part + 1e-12, (i, options[i], share[i], part)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab,pad", [(1, 0), (2, 1), (7, 0), (500, 3), (4099, 0), (20011, 5)])
def test_options(dtype, vocab, pad):
    rng = np.random.default_rng(vocab)
    wide = torch.full((len(OPTIONS), vocab + pad), 60.0, dtype=dtype, device="cuda")
    logits = wide[:, :vocab]
    logits.copy_(torch.from_numpy(rng.standard_normal((len(OPTIONS), vocab)) * 3))
    compare(logits, OPTIONS, rng)


@pytest.mark.parametrize("dtype", TYPES)
def test_a_large_vocabulary(dtype):
    rng = np.random.default_rng(8)
    options = [dict(), dict(top_k=50, top_p=0.95, temperature=0.8), dict(top_p=0.9), dict(min_p=0.05), dict(top_k=5000)]
    logits = torch.from_numpy(rng.standard_normal((len(options), 128256)) * 3).to(dtype).cuda()
    compare(logits, options, rng, tries=2)


@pytest.mark.parametrize("dtype", TYPES)
def test_equal_logits(dtype):
    """Whole groups of equal words at the cut: the lowest stay."""
    rng = np.random.default_rng(6)
    values = np.array([-2.0, 0.0, -0.0, 1.5, 1.5, 3.0])
    options = [o for o in OPTIONS for _ in range(2)] + [dict(top_k=k) for k in (2, 100, 333, 1999)] + [dict(top_p=p) for p in (0.01, 0.5, 0.75)]
    logits = torch.from_numpy(rng.choice(values, (len(options), 2000))).to(dtype).cuda()
    logits[0] = 1.0
    logits[1] = -5.0
    options[1] = dict(top_k=17)
    compare(logits, options, rng)


@pytest.mark.parametrize("dtype", TYPES)
def test_words_that_take_no_part(dtype):
    rng = np.random.default_rng(7)
    logits = torch.from_numpy(rng.standard_normal((8, 3001)) * 2).to(dtype).cuda()
    logits[0] = -math.inf
    logits[1] = math.nan
    logits[2] = -math.inf
    logits[2, 1234] = -3.0
    logits[3, ::2] = math.nan
    logits[4, 10:2990] = -math.inf
    logits[5, 77], logits[5, 2000] = math.inf, math.inf
    logits[6] = -math.inf
    logits[6, 3000] = math.inf
    options = [dict(), dict(top_k=5), dict(top_p=0.5), dict(top_k=20, top_p=0.9), dict(top_k=3000), dict(), dict(top_k=4, min_p=0.5), dict(temperature=0.0)]
    logits[7, :100] = math.nan
    compare(logits, options, rng)
    token, share = call(logits, [0.5] * 8, [dict(temperature=0.0)] * 8)
    assert token[0] == token[1] == -1 and share[0] == share[1] == 0 and token[2] == 1234 and token[5] == 77 and token[6] == 3000


def test_parameters_at_and_beyond_their_ends():
    rng = np.random.default_rng(3)
    logits = torch.from_numpy(rng.standard_normal((1, 999))).cuda().float()
    x = logits.double().cpu().numpy()[0]
    every = sm.stays(list(x))
    best = int(np.argmax(x))
    first, last = 0, 998

    def one(u=0.5, **options):
        token, share = call(logits, [u], [options])
        return token[0], share[0]

    want = sm.choose(every, 0.5)[0]
    for options in (dict(top_k=-3), dict(top_k=0), dict(top_k=10 ** 9), dict(top_p=1.0), dict(top_p=7.0), dict(top_p=math.nan), dict(min_p=0.0), dict(min_p=-1.0), dict(min_p=math.nan)):
        assert one(**options)[0] == want, options
    for options in (dict(top_p=0.0), dict(top_p=-1.0), dict(min_p=1.0), dict(min_p=50.0), dict(temperature=-1.0), dict(temperature=math.nan), dict(temperature=1e-30), dict(top_k=1)):
        assert one(**options) == (best, 1.0), options
    assert one(0.0)[0] == one(-2.0)[0] == one(math.nan)[0] == first
    assert one(1.0)[0] == one(5.0)[0] == one(math.inf)[0] == last
    # An infinite temperature makes all words alike.
    assert one((500 + 0.5) / 999, temperature=math.inf)[0] == 500


def test_all_words_are_drawn_as_often_as_they_should():
    """A thousand random numbers, evenly spaced, through one row: every word as often as its share says, to one."""
    x = torch.linspace(-2, 1, 13).cuda()
    n = 1000
    random = (torch.arange(n, device="cuda") + 0.5) / n
    token = torch.empty(n, dtype=torch.int32, device="cuda")
    wq.sample_logits(x.expand(n, 13).contiguous(), random, token)
    count = torch.bincount(token.long(), minlength=13).double().cpu()
    assert bool(((count - torch.softmax(x.double(), 0).cpu() * n).abs() <= 1).all())


def test_results_do_not_depend_on_the_batch_or_the_run():
    g = torch.Generator(device="cuda").manual_seed(3)
    logits = torch.randn((40, 50021), generator=g, device="cuda") * 3
    random = torch.rand(40, generator=g, device="cuda")
    p = torch.full((40,), 0.93, device="cuda")
    token, again, one = (torch.empty(40, dtype=torch.int32, device="cuda") for _ in range(3))
    wq.sample_logits(logits, random, token, top_p=p)
    for _ in range(3):
        wq.sample_logits(logits, random, again, top_p=p)
        assert torch.equal(token, again)
    for i in range(40):
        wq.sample_logits(logits[i:i + 1], random[i:i + 1], one[i:i + 1], top_p=p[i:i + 1])
    assert torch.equal(token, one)


def test_captured_and_replayed():
    logits = torch.zeros((5, 30000), dtype=torch.float16, device="cuda")
    random, p = torch.zeros(5, device="cuda"), torch.full((5,), 0.9, device="cuda")
    k = torch.full((5,), 100, dtype=torch.int32, device="cuda")
    token = torch.empty(5, dtype=torch.int32, device="cuda")
    workspace = wq.sample_workspace(logits)

    def step():
        wq.sample_logits(logits, random, token, top_k=k, top_p=p, workspace=workspace)

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in range(3):
        g = torch.Generator(device="cuda").manual_seed(seed)
        logits.copy_(torch.randn(logits.shape, generator=g, device="cuda") * 3)
        random.copy_(torch.rand(5, generator=g, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        kept = token.clone()
        step()
        assert torch.equal(kept, token)
