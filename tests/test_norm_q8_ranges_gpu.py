"""mb_rmsnorm_q8 where fp32 ends on the way: residuals and norms that are subnormal, weights that lift them again, rows whose
elements span more than fp32's squares. Values and scales are those of the definition in 64 bits (oracle/serve.py): the
norm carries 2^-44, so an element differs only where it is that near to a border between two 8-bit values."""
import numpy as np
import pytest
import torch

from oracle import serve
from paper_2401_13660_gb300 import mbscan as mb

from _parity import to_np

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _check(residual, w, eps=1e-5, add=None):
    rows, width = residual.shape
    q = torch.full((rows, width), 0x55, dtype=torch.uint8, device=DEV)
    s = torch.full((rows, serve.stride(width)), 0x55, dtype=torch.uint8, device=DEV)
    mb.mb_rmsnorm_q8(residual, w, q, s, add=add, eps=eps)
    rq, rs = serve.quantize(serve.rmsnorm(to_np(residual), to_np(w), float(np.float32(eps))), 1)
    assert np.array_equal(s.cpu().numpy(), rs)
    got = serve.e4m3_values(q.cpu().numpy())
    assert np.array_equal(got, rq), (np.argwhere(got != rq)[:5], int((got != rq).sum()))


def _rnd(rows, width, seed):
    return torch.randn(rows, width, device=DEV, generator=torch.Generator(device=DEV).manual_seed(seed))


# few rows (a warp to a block) and many (four), and rows that are read again
SIZES = [(5, 640), (700, 1024), (2, 20496)]


@pytest.mark.parametrize("rows, width", SIZES)
@pytest.mark.parametrize("tiny, weight", [(1e-43, 1e38), (1e-40, 1e30), (1e-38, 1e20), (1e-35, 1e38), (1e-43, 1e10)])
def test_weights_lift_what_is_subnormal(rows, width, tiny, weight):
    residual = _rnd(rows, width, 1)
    residual[:, 128:512] *= tiny
    w = torch.rand(width, device=DEV) + 0.5
    w[128:512] *= weight
    _check(residual, w)


@pytest.mark.parametrize("rows, width", SIZES)
@pytest.mark.parametrize("large, small, weight", [(1e30, 1e-10, 1e36), (1e25, 1e-30, 1e38), (1e37, 1e-3, 1e38), (1e19, 1e-20, 1e30)])
def test_rows_of_a_wide_span(rows, width, large, small, weight):
    """What the small elements lose next to the large ones' squares is not lost from themselves."""
    residual = _rnd(rows, width, 2)
    residual[:, :128] *= large
    residual[:, 128:] *= small
    w = torch.rand(width, device=DEV) + 0.5
    w[128:] *= weight
    _check(residual, w)


@pytest.mark.parametrize("rows, width", SIZES)
@pytest.mark.parametrize("weight", [1e-35, 1e-38, 1e-40, 1e-42])
def test_norms_below_the_range(rows, width, weight):
    """The lowest scale is 2^-126: below 2^-136 there is nothing, above it every step is rounded to nearest."""
    _check(_rnd(rows, width, 3), _rnd(1, width, 4)[0] * weight)


@pytest.mark.parametrize("rows, width", SIZES)
def test_one_weight_among_others(rows, width):
    """A large weight at an element that is nothing, or next to nothing, beside ordinary ones."""
    residual = _rnd(rows, width, 5)
    residual[:, 3], residual[:, 200] = 0.0, 1e-44
    w = torch.rand(width, device=DEV) + 0.5
    w[3], w[200] = 3e38, 2e38
    _check(residual, w, add=_rnd(rows, width, 6).where(torch.arange(width, device=DEV) % 197 != 3, 0.0))
    _check(torch.zeros(rows, width, device=DEV), w)


@pytest.mark.parametrize("rows, width", SIZES)
@pytest.mark.parametrize("scale, weight", [(1e-44, 1.0), (1e-42, 1e30), (1e-38, 1e-5), (1e38, 1e10), (1e30, 1e-30)])
def test_rows_at_the_ends_without_eps(rows, width, scale, weight):
    residual = (_rnd(rows, width, 7).clamp(-3, 3) * scale)
    residual[:, 0] = scale   # no row of zeros
    _check(residual, (torch.rand(width, device=DEV) + 0.5) * weight, eps=0.0)


@pytest.mark.parametrize("rows, width", SIZES)
@pytest.mark.parametrize("weight", [2.0 ** -17, 2.0 ** -20, 2.0 ** 17, 2.0 ** 60, 2.0 ** 64, 2.0 ** 66, 2.0 ** 100])
def test_norms_of_every_size(rows, width, weight):
    """Across the limits within which fp32 is taken to hold what it takes."""
    _check(_rnd(rows, width, 8), (_rnd(1, width, 9)[0].abs() + 0.1) * weight)


@pytest.mark.parametrize("rows, width", SIZES)
def test_an_infinity_leaves_zeros_beside_it(rows, width):
    residual, w = _rnd(rows, width, 10), torch.rand(width, device=DEV) + 0.5
    residual[1, 5], residual[0, 130] = float("inf"), -float("inf")
    q = torch.empty(rows, width, dtype=torch.uint8, device=DEV)
    s = torch.empty(rows, serve.stride(width), dtype=torch.uint8, device=DEV)
    mb.mb_rmsnorm_q8(residual, w, q, s)
    v = serve.dequantize(q.cpu().numpy(), s.cpu().numpy(), 1)
    assert np.isnan(v[1, 5]) and np.isnan(v[0, 130]) and np.isnan(v).sum() == 2
    v[1, 5] = v[0, 130] = 0.0
    assert not v[:2].any() and (rows == 2 or v[2:].any())
