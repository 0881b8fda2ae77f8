"""fp32 results of the training operators to the precision of fp32, where a
short cut through the special function unit shows.

Bounds, u = 2^-24, derived before the first run. Losses: where all other logits
are 30 and more below the largest, which is 0, the sum of exponentials is 1 to
the last bit and the differences are exact, so a gradient is one exponential: 4 u
of the unit's 2^x, u of each of the three roundings behind it (the correction of
its argument, their product, the row's factor); twice over for slack. Rows of
equal logits: exponentials of 1 and their sum are exact, so the gradient is the
correctly rounded quotient."""
import numpy as np
import pytest
import torch

from paper_2401_13660_gb300 import mbscan as mb

from _parity import to_np

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24

# every kernel: several rows to a warp, a warp, a row kept in registers, read twice, by several CTAs
ROWS = [(5, 8), (300, 128), (70, 256), (9, 250), (7, 700), (6, 1024), (20, 5000), (3, 5001), (310, 8200), (2, 20001), (1, 40000)]


@pytest.mark.parametrize("n, V", ROWS)
def test_gradients_far_below_the_largest_logit(n, V):
    g = torch.Generator(device=DEV).manual_seed(n + V)
    logits = -torch.randint(30 * 64, 85 * 64, (n, V), device=DEV, generator=g).float() / 64
    tgt = torch.randint(0, V, (n,), device=DEV, generator=g)
    logits.scatter_(1, tgt[:, None], 0.0)
    loss, d = torch.empty(n, device=DEV), torch.empty_like(logits)
    mb.mb_cross_entropy(logits, tgt, loss, d)
    ref, got = np.exp(to_np(logits)), to_np(d)
    off = np.abs(got / ref - 1)
    np.put_along_axis(off, tgt.cpu().numpy()[:, None], 0.0, 1)
    assert off.max() <= 14 * U, off.max() / U
    assert (loss == 0).all() and (d.gather(1, tgt[:, None]) == 0).all()


@pytest.mark.parametrize("n, V", [(300, 512), (300, 510), (900, 1024), (900, 1023), (200, 1028), (200, 5001), (120, 8200), (40, 20001), (3, 40000)])
def test_gradients_of_equal_logits_are_rounded_once(n, V):
    logits = torch.full((n, V), -float("inf"), device=DEV)
    for r in range(n):
        logits[r, :r + 2] = 1.5
    tgt = torch.zeros(n, dtype=torch.int32, device=DEV)
    loss, d = torch.empty(n, device=DEV), torch.empty_like(logits)
    mb.mb_cross_entropy(logits, tgt, loss, d, scale=0.7)
    want = np.float32(0.7) / np.arange(2, n + 2, dtype=np.float32)
    assert np.array_equal(d[:, 1].cpu().numpy(), want)
    assert all((d[r, 1:r + 2] == d[r, 1]).all() and (d[r, r + 2:] == 0).all() for r in range(n))
