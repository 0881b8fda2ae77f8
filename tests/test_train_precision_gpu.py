"""fp32 results of the training operators to the precision of fp32, where a
short cut through the special function unit shows.

Bounds, u = 2^-24, derived before the first run. Losses: where all other logits
are 30 and more below the largest, which is 0, the sum of exponentials is 1 to
the last bit and the differences are exact, so a gradient is one exponential: 4 u
of the unit's 2^x, u of each of the three roundings behind it (the correction of
its argument, their product, the row's factor); twice over for slack. Rows of
equal logits: exponentials of 1 and their sum are exact, so the gradient is the
correctly rounded quotient. SiLU of one tap of weight 1, so that p = x exactly:
7 u of the exponential as above (bf16, whose exponent is a plain product: (1.5 |p| +
4) u), u of 1 + e, 2 u of the unit's reciprocal, 2 u of products, twice over; its
slope s (1 + p (1 - s)) two more roundings and, at p <= -5, no cancellation. What
is stored lies between the roundings of the ends of that interval. Below 2^-126 a sigmoid is good to 2^-150, times |p| < 89. Past p = -88.72 e^-p overflows
and SiLU, there above -2.7e-37, may be zero."""
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


def _one_tap(x):
    w = torch.zeros(x.shape[2], 4, device=DEV)
    w[:, 3] = 1
    out = mb.mb_conv1d(x, w, torch.empty_like(x))
    dx = mb.mb_conv1d_backward(x, w, torch.ones_like(x))["dx"]
    return to_np(out), to_np(dx)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_silu_down_to_where_its_exponential_overflows(dtype):
    p = torch.linspace(-88.7, 40, 4096, device=DEV).to(dtype).view(2, 128, 16)
    out, dx = _one_tap(p)
    x = to_np(p)
    e = (1.5 * np.abs(x) + 4) * U if dtype == torch.bfloat16 else 7 * U

    def within(got, ref, rel):
        off = 2 * rel * np.abs(ref) + 90 * 2.0 ** -149
        lo, hi = (to_np(torch.from_numpy(ref + sign * off).to(dtype)) for sign in (-1, 1))
        return (lo <= got) & (got <= hi)
    assert within(out, x / (1 + np.exp(-x)), e + 5 * U).all()
    s = 1 / (1 + np.exp(-x))
    assert within(dx, s * (1 + x * (1 - s)), e + 7 * U)[x <= -5].all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_silu_beyond(dtype):
    p = torch.tensor([-89.0, -95.0, -99.5, -100.5, -130.0, -1e4, -1e30, -3e38, 90.0, 99.5, 100.5, 130.0, 1e4, 1e30, 3e38, 0.0],
                     device=DEV).to(dtype).view(1, 1, 16)
    out, dx = _one_tap(p)
    x = to_np(p)
    assert np.all(np.abs(out[x < 0]) <= 2.7e-37) and np.all(np.abs(dx[x < 0]) <= 2.7e-37)
    assert np.array_equal(out[x >= 0], x[x >= 0]) and np.all(dx[x > 0] == 1) and dx.flat[-1] == 0.5
    p.flatten()[:3] = torch.tensor([float("nan"), float("-inf"), float("inf")], device=DEV).to(dtype)
    out, dx = _one_tap(p)
    assert np.isnan(out.flat[0]) and np.isnan(dx.flat[0]) and out.flat[2] == np.inf
    assert np.isfinite(out.flat[3:]).all() and np.isfinite(dx.flat[3:]).all()
