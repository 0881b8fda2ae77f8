"""mb_sample against the definition in 64 bits (oracle/serve.py), row by row.

Weights are within 2^-31 of their value, so the token is that of exact arithmetic unless u, top_p or min_p is within two
such errors (2^-30, relative) of a border between two; the probability of a token is a quotient of two such, rounded to fp32 three
times: 2^-22."""
import itertools

import numpy as np
import pytest
import torch

from oracle import serve
from paper_2401_13660_gb300 import mbscan as mb

from _parity import to_np

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
MOST = {"f32": float(np.finfo(np.float32).max), "bf16": float(np.uint32(0x7f7f0000).view(np.float32))}
NEAR = 2.0 ** -30


def _sample(logits, u, kind=torch.int64, **settings):
    n = logits.shape[0]
    tokens = torch.full((n,), -7, dtype=kind, device=DEV)
    prob = torch.full((n,), float("nan"), device=DEV)
    mb.mb_sample(logits, u, tokens, prob=prob, **settings)
    without = torch.empty_like(tokens)
    mb.mb_sample(logits, u, without, **settings)
    assert torch.equal(tokens, without)
    return tokens.cpu().numpy(), prob.cpu().numpy()


def _check(logits, u, tokens, prob, dtype, **settings):
    l, u = to_np(logits), to_np(u)
    s = {k: to_np(v) for k, v in settings.items()}
    for r in range(l.shape[0]):
        mine = {k: (int(v[r]) if k == "top_k" else float(v[r])) for k, v in s.items()}
        want, p = serve.sample(l[r], u[r], most=MOST[dtype], **mine)
        if tokens[r] != want:
            near = set()
            for du, dp, dm in itertools.product((-NEAR, 0, NEAR), repeat=3):
                moved = dict(mine)
                if "top_p" in moved:
                    moved["top_p"] *= 1 + dp
                if "min_p" in moved:
                    moved["min_p"] *= 1 + dm
                near.add(serve.sample(l[r], u[r] + du, most=MOST[dtype], **moved)[0])
            assert tokens[r] in near, (r, tokens[r], want, mine, u[r])
        else:
            assert abs(prob[r] - p) <= 2.0 ** -22 * p, (r, prob[r], p, mine)


def _settings(n, g, which):
    def choose(values, dtype):
        return torch.tensor(values, device=DEV, dtype=dtype)[torch.randint(0, len(values), (n,), device=DEV, generator=g)]
    every = dict(temperature=choose([0.0, 0.3, 0.7, 1.0, 2.5], torch.float32), top_k=choose([0, 1, 2, 7, 40, 300, 5000], torch.int32),
                 top_p=choose([0.1, 0.5, 0.9, 0.99, 1.0], torch.float32), min_p=choose([0.0, 0.01, 0.2, 1.0], torch.float32))
    return {k: every[k] for k in which}


def _logits(n, vocab, dtype, g, spread=2.0):
    l = spread * torch.randn(n, vocab, device=DEV, generator=g)
    l[torch.rand(n, vocab, device=DEV, generator=g) < 0.05] = -float("inf")
    l[:, vocab // 2] = 1.0
    return l.to(TYPES[dtype])


SETS = [(), ("temperature",), ("top_k",), ("top_p",), ("min_p",), ("top_k", "top_p"), ("temperature", "top_k", "top_p", "min_p")]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("which", SETS, ids="-".join)
@pytest.mark.parametrize("n, vocab", [(1, 1), (40, 2), (64, 7), (200, 255), (300, 256), (700, 200), (64, 257), (40, 1000), (24, 4099)])
def test_draw(n, vocab, which, dtype):
    g = torch.Generator(device=DEV).manual_seed(n + vocab)
    logits = _logits(n, vocab, dtype, g)
    u = torch.rand(n, device=DEV, generator=g)
    settings = _settings(n, g, which)
    tokens, prob = _sample(logits, u, torch.int32 if n % 2 else torch.int64, **settings)
    _check(logits, u, tokens, prob, dtype, **settings)


@pytest.mark.parametrize("vocab, dtype", [(32001, "bf16"), (50257, "f32"), (130000, "bf16"), (200003, "f32"), (600007, "f32")])
def test_large_vocabularies(vocab, dtype):
    g = torch.Generator(device=DEV).manual_seed(vocab)
    n = 5
    logits = _logits(n, vocab, dtype, g)
    u = torch.rand(n, device=DEV, generator=g)
    for which in (("top_p",), ("top_k", "top_p", "min_p", "temperature"), ()):
        settings = _settings(n, g, which)
        tokens, prob = _sample(logits, u, **settings)
        _check(logits, u, tokens, prob, dtype, **settings)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [256, 5000, 20000])
def test_ties_go_to_the_lower_index(vocab, dtype):
    """Few different logits, or one: the tokens that top_k and top_p keep end among equals, also among more than are ranked
    one against the other. Masses are multiples of equal weights: u and top_p fall on borders, and are met exactly."""
    g = torch.Generator(device=DEV).manual_seed(vocab)
    n = 8
    logits = torch.randint(0, 2, (n, vocab), device=DEV, generator=g).float()
    logits[4:] = 3.0
    logits = logits.to(TYPES[dtype])
    for top_k, top_p in ((0, 0.5), (0, 0.25), (vocab // 2, 1.0), (vocab * 3 // 4, 0.75), (3, 1.0), (0, 1e-30)):
        for step in (0.0, 0.125, 0.5, 1.0 - 2.0 ** -24):
            u = torch.full((n,), step, device=DEV)
            settings = dict(top_k=torch.full((n,), top_k, dtype=torch.int32, device=DEV), top_p=torch.full((n,), top_p, device=DEV))
            tokens, prob = _sample(logits, u, **settings)
            _check(logits, u, tokens, prob, dtype, **settings)
            equal = vocab if top_k == 0 else top_k   # of the rows of one logit: the first of them
            left = max(1, int(np.ceil(float(np.float32(top_p)) * equal))) if top_p < 1 else equal
            assert (tokens[4:] == int(np.floor(float(np.float32(step)) * left))).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [9, 256, 3000])
def test_masked_infinite_and_missing_numbers(vocab, dtype):
    inf, nan = float("inf"), float("nan")
    g = torch.Generator(device=DEV).manual_seed(5)
    l = torch.randn(9, vocab, device=DEV, generator=g)
    l[0] = -inf                       # nothing left
    l[1] = nan
    l[2], l[2, vocab - 2] = -inf, -5.0   # one token
    l[3, 4], l[3, 6] = inf, inf       # share the mass
    l[4, ::2] = nan
    l[5] = -3e38                      # far from 0, all the same
    l[6], l[6, 3] = -3e38, 3e38
    l[7, :4] = -0.0
    l[7, 4:8] = 0.0
    l[7, 8:] = -1.0
    l[8, 0] = inf
    logits = l.to(TYPES[dtype])
    for which in ((), ("top_p",), ("top_k", "top_p"), ("temperature", "top_k", "min_p")):
        for u in (0.0, 0.3, 0.9):
            u = torch.full((9,), u, device=DEV)
            settings = _settings(9, g, which)
            tokens, prob = _sample(logits, u, **settings)
            assert tokens[0] == tokens[1] == -1 and prob[0] == prob[1] == 0
            assert tokens[2] == vocab - 2 and prob[2] == 1 and tokens[8] == 0
            _check(logits, u, tokens, prob, dtype, **settings)


@pytest.mark.parametrize("vocab", [256, 700])
def test_settings_at_their_ends(vocab):
    g = torch.Generator(device=DEV).manual_seed(1)
    logits = torch.randn(12, vocab, device=DEV, generator=g)
    best = logits.argmax(1).cpu().numpy()
    f = lambda *v: torch.tensor(v, device=DEV)   # noqa: E731
    u = torch.rand(12, device=DEV, generator=g)
    base, _ = _sample(logits, u)
    inf, nan = float("inf"), float("nan")
    tokens, prob = _sample(logits, u, temperature=f(0.0, -1.0, nan, 1e-30, 1e-45, inf, 1.0, 1.0, 3e38, 1e-6, 1.0, 1.0))
    assert (tokens[[0, 1, 2, 3, 4, 9]] == best[[0, 1, 2, 3, 4, 9]]).all() and (prob[:5] == 1).all()
    assert (tokens[[5, 8]] == np.floor(u.cpu().numpy()[[5, 8]].astype(np.float64) * vocab)).all()   # all the same
    assert (tokens[[6, 7, 10, 11]] == base[[6, 7, 10, 11]]).all()
    tokens, _ = _sample(logits, u, top_p=f(0.0, -1.0, 1e-45, nan, 1.0, 2.0, inf, -inf, 1.0, 1.0, 1.0, 1.0))
    assert (tokens[[0, 1, 2, 7]] == best[[0, 1, 2, 7]]).all() and (tokens[[3, 4, 5, 6, 8]] == base[[3, 4, 5, 6, 8]]).all()
    tokens, _ = _sample(logits, u, min_p=f(1.0, 2.0, inf, 0.0, -1.0, nan, -inf, 1e-45, 1.0, 1.0, 1.0, 1.0))
    assert (tokens[[0, 1, 2, 8]] == best[[0, 1, 2, 8]]).all() and (tokens[[3, 4, 5, 6, 7]] == base[[3, 4, 5, 6, 7]]).all()
    k = torch.tensor([1, 0, -5, vocab, vocab + 1, 2 ** 31 - 1, -2 ** 31, 1, 1, 1, 1, 1], dtype=torch.int32, device=DEV)
    tokens, _ = _sample(logits, u, top_k=k)
    assert (tokens[[0, 7, 8]] == best[[0, 7, 8]]).all() and (tokens[1:7] == base[1:7]).all()
    first, _ = _sample(logits, f(0.0, -1.0, nan, -inf, 0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 0.0))
    last, _ = _sample(logits, f(1.0, 2.0, inf, 1.0, 1.0, 1.0, 1.0, 1.0, 1.0, 1.0, 1.0, 1.0))
    assert not first.any() and (last == vocab - 1).all()


def test_frequencies():
    """65536 draws by evenly spread numbers: every token as often as its share of the mass says, but for the two ends."""
    n, vocab = 65536, 256
    logits = torch.randn(vocab, device=DEV, generator=torch.Generator(device=DEV).manual_seed(2))
    u = (torch.arange(n, device=DEV) + 0.5) / n
    tokens, prob = _sample(logits.repeat(n, 1), u)
    p = torch.softmax(logits.double(), 0).cpu().numpy()
    assert np.abs(np.bincount(tokens, minlength=vocab) - n * p).max() <= 2
    assert np.abs(prob - p[tokens]).max() <= 2.0 ** -22


def test_ties_in_a_row_that_does_not_fit():
    """Read from memory in every pass, equals across the parts of a cluster."""
    n, vocab = 3, 600001
    logits = torch.full((n, vocab), 1.5, device=DEV)
    logits[0, ::2] = 1.0
    u = torch.full((n,), 0.75, device=DEV)
    for top_k, top_p in ((0, 0.5), (400000, 1.0), (450001, 0.25), (7, 1.0)):
        settings = dict(top_k=torch.full((n,), top_k, dtype=torch.int32, device=DEV), top_p=torch.full((n,), top_p, device=DEV))
        tokens, prob = _sample(logits, u, **settings)
        _check(logits, u, tokens, prob, "f32", **settings)


def test_offsets_beyond_32_bits():
    n, vocab = 2047, 1048573
    logits = torch.zeros(n, vocab, dtype=torch.bfloat16, device=DEV)
    at = torch.randint(0, vocab, (n,), device=DEV)
    logits.scatter_(1, at[:, None], 30.0)
    u = torch.rand(n, device=DEV)
    for settings in ({}, dict(top_p=torch.full((n,), 0.5, device=DEV)), dict(temperature=torch.zeros(n, device=DEV))):
        tokens = mb.mb_sample(logits, u, **settings)
        assert torch.equal(tokens, at)


def test_no_rows():
    assert mb.mb_sample(torch.empty(0, 256, device=DEV), torch.empty(0, device=DEV)).shape == (0,)
