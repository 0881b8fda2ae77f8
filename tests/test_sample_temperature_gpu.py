"""mb_sample at temperatures near the lower end of fp32: the scale log2(e) / T stays as exact as elsewhere down to T = 2^-127,
which is where lower ones are taken to be. Logits are a few T apart, so their weights matter.

Weights are within 2^-31 of their value and the probability is a quotient of two, rounded to fp32 three times: 2^-22."""
import numpy as np
import pytest
import torch

from oracle import serve
from paper_2401_13660_gb300 import mbscan as mb

from _parity import to_np

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
LEAST = 2.0 ** -127


@pytest.mark.parametrize("vocab", [2, 200, 700, 5000])
@pytest.mark.parametrize("first", [8.48e-39, 4.3e-39 * 1.4, 1.2e-38, 1.1e-37, 2.0 ** -127, 2.0 ** -130, 2.0 ** -149])
def test_cold_draws(vocab, first):
    n = 48
    t = np.float32(first) + np.arange(n).astype(np.float32) * np.float32(2.0 ** -149)   # neighbours of it
    steps = np.minimum(np.arange(vocab) * 16.0 / vocab + 0.5, 16.0)
    logits = (-np.maximum(t, LEAST)[:, None].astype(np.float64) * np.log(2.0) * steps).astype(np.float32)
    logits[:, 0] = 0.0
    u = np.full(n, 1.0, np.float32)   # the last token
    u[::3] = np.linspace(0.0, 0.9, len(u[::3]))
    tokens, prob = torch.empty(n, dtype=torch.int64, device=DEV), torch.empty(n, device=DEV)
    put = lambda x: torch.from_numpy(x).to(DEV)   # noqa: E731
    mb.mb_sample(put(logits), put(u), tokens, temperature=put(t), prob=prob)
    got, p = tokens.cpu().numpy(), to_np(prob)
    for r in range(n):
        cold = max(float(t[r]), LEAST)
        near = {serve.sample(logits[r], float(u[r]) + d, temperature=cold)[0] for d in (-2.0 ** -30, 0.0, 2.0 ** -30)}
        assert got[r] in near
        w = np.exp(logits[r].astype(np.float64) / cold)
        want = w[got[r]] / w.sum()
        assert abs(p[r] - want) <= 2.0 ** -22 * want, (r, got[r], p[r], want)
