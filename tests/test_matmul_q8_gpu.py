"""mb_matmul_q8 against the product in 64 bits (oracle/serve.py).

Products of e4m3 numbers and powers of two are exact; the sum of K of them in fp32 is within K 2^-23 of the sum of
their magnitudes (a unit in the last place each, whichever way the tensor core rounds), and the result is rounded once:
half a step, 2^-8 in bf16, 2^-24 in fp32."""
import numpy as np
import pytest
import torch

from oracle import serve
from paper_2401_13660_gb300 import mbscan as mb

from _parity import to_np

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def _matrix(rows, width, block_rows, seed, spread=4):
    g = torch.Generator(device=DEV).manual_seed(seed + 7 * rows + width)
    q = (torch.randn(rows, width, device=DEV, generator=g) * 100).clamp(-448, 448).to(torch.float8_e4m3fn)
    s = torch.randint(127 - spread, 128 + spread, (-(-rows // block_rows), serve.stride(width)), device=DEV, generator=g)
    return q, s.to(torch.uint8)


def _check(a, sa, w, sw, out, dtype):
    got = to_np(out)
    rows, n = a.shape[0], w.shape[0]
    if got.ndim == 3:
        got = got.transpose(1, 0, 2).reshape(rows, n)
    want, size = serve.matmul(*(t.view(torch.uint8).cpu().numpy() for t in (a, sa, w, sw)))
    assert np.array_equal(np.isnan(got), np.isnan(want))
    bound = a.shape[1] * 2.0 ** -23 * size * (1 + HALF[dtype]) + HALF[dtype] * np.abs(want)
    bad = np.abs(got - want) > bound
    assert not bad.any(), (np.argwhere(bad)[:5], got[bad][:5], want[bad][:5])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows, n, width", [
    (1, 8, 16), (1, 128, 128), (16, 128, 128), (17, 136, 144), (1, 1024, 1024), (5, 264, 512), (128, 256, 640), (129, 256, 384),
    (240, 128, 256), (241, 128, 256), (255, 1000, 400), (256, 512, 2304), (1003, 520, 1552), (3, 4608, 64), (500, 8, 4608),
    (2, 2304, 4608), (64, 2304, 4608), (33, 128, 8192),
    (1025, 264, 272), (1500, 136, 640), (2047, 1032, 1040), (4100, 512, 128), (1200, 2304, 512)])
def test_product(rows, n, width, dtype):
    a, sa = _matrix(rows, width, 1, 1)
    w, sw = _matrix(n, width, 128, 2)
    out = torch.full((rows, n), float("nan"), dtype=TYPES[dtype], device=DEV)
    ws = torch.zeros(256, dtype=torch.uint8, device=DEV)
    mb.mb_matmul_q8(a, sa, w, sw, out, ws=ws)
    assert mb.mb_check(ws)[0] == mb.MB_OK
    _check(a, sa, w, sw, out, dtype)
    again = torch.empty_like(out)
    mb.mb_matmul_q8(a, sa, w, sw, again)
    assert torch.equal(out, again)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [2, 31, 64, 100, 200, 250, 320, 384])
@pytest.mark.parametrize("n, width", [(128, 8192), (264, 2304), (1024, 4608), (2304, 4608)])
def test_sums_in_parts(rows, n, width, dtype):
    """Few tiles: two, four or eight parts of a sum, of tiles of every height, with rows missing in the last."""
    a, sa = _matrix(rows, width, 1, 11)
    w, sw = _matrix(n, width, 128, 12)
    out = torch.full((rows, n), float("nan"), dtype=TYPES[dtype], device=DEV)
    mb.mb_matmul_q8(a, sa, w, sw, out)
    _check(a, sa, w, sw, out, dtype)
    again = torch.empty_like(out)
    mb.mb_matmul_q8(a, sa, w, sw, again)
    assert torch.equal(out, again)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows, n, width", [(65, 19720, 144), (100, 19592, 640), (225, 10008, 272), (385, 6664, 400),
                                            (4096, 776, 4608), (3001, 520, 4112), (64, 19720, 144), (500, 2304, 16384)])
def test_wide_products(rows, n, width, dtype):
    """Pairs of CTAs, of tiles low and high, the last ones ragged both ways."""
    a, sa = _matrix(rows, width, 1, 13)
    w, sw = _matrix(n, width, 128, 14)
    out = torch.full((rows, n), float("nan"), dtype=TYPES[dtype], device=DEV)
    mb.mb_matmul_q8(a, sa, w, sw, out)
    _check(a, sa, w, sw, out, dtype)


@pytest.mark.parametrize("rows, parts", [(1, 2), (37, 3), (300, 2), (1100, 2)])
def test_groups_of_columns_come_apart(rows, parts):
    a, sa = _matrix(rows, 1040, 1, 3)
    w, sw = _matrix(parts * 384, 1040, 128, 4)
    whole, apart = torch.empty(rows, parts * 384, device=DEV), torch.empty(parts, rows, 384, device=DEV)
    mb.mb_matmul_q8(a, sa, w, sw, whole)
    mb.mb_matmul_q8(a, sa, w, sw, apart)
    assert torch.equal(whole, apart.transpose(0, 1).reshape(rows, -1))


@pytest.mark.parametrize("rows, n, width", [(3, 264, 640), (300, 264, 640), (1100, 264, 640), (2, 128, 4608)])
def test_what_is_no_number_stays_in_its_sums(rows, n, width):
    """NaN among the values, and scales that are none."""
    a, sa = _matrix(rows, width, 1, 5)
    w, sw = _matrix(n, width, 128, 6)
    a.view(torch.uint8)[1, 130] = 0x7f
    sa[rows - 1, 4] = 255
    w.view(torch.uint8)[n - 1, 3] = 0xff
    out = torch.empty(rows, n, device=DEV)
    mb.mb_matmul_q8(a, sa, w, sw, out)
    nan = out.isnan()
    assert nan[1].all() and nan[rows - 1].all() and nan[:, n - 1].all()
    assert int(nan.sum()) == (1 if rows == 2 else 2) * n + rows - (1 if rows == 2 else 2)
    _check(a, sa, w, sw, out, "f32")


@pytest.mark.parametrize("rows", [2, 200, 1200])
def test_scales_at_their_ends(rows):
    """The smallest and largest scales: products below and above fp32's range are zeros and infinities."""
    a, w = (torch.full((n, 256), 1.0, device=DEV).to(torch.float8_e4m3fn) for n in (rows, 256))
    out = torch.empty(rows, 256, device=DEV)
    for x, y, want in ((0, 254, 256.0), (254, 0, 256.0), (127, 127, 256.0), (1, 1, 0.0), (254, 254, float("inf")), (64, 190, 256.0)):
        sa = torch.full((rows, 4), x, dtype=torch.uint8, device=DEV)
        sw = torch.full((2, 4), y, dtype=torch.uint8, device=DEV)
        mb.mb_matmul_q8(a, sa, w, sw, out)
        assert (out == want).all(), (x, y, out[0, 0])


def test_nothing_behind_the_result():
    for rows, n in ((1, 8), (17, 264), (300, 136), (1500, 264)):
        a, sa = _matrix(rows, 144, 1, 7)
        w, sw = _matrix(n, 144, 128, 8)
        room = torch.full((rows * n + 4096,), 7.0, dtype=torch.bfloat16, device=DEV)
        mb.mb_matmul_q8(a, sa, w, sw, room[:rows * n].view(rows, n))
        assert (room[rows * n:] == 7.0).all() and not (room[:rows * n] == 7.0).all()


def test_sums_of_nothing():
    a, w = (torch.empty(n, 0, dtype=torch.uint8, device=DEV) for n in (5, 16))
    out = torch.full((5, 16), 3.0, device=DEV)
    mb.mb_matmul_q8(a, torch.empty(5, 0, dtype=torch.uint8, device=DEV), w, torch.empty(1, 0, dtype=torch.uint8, device=DEV), out)
    assert not out.any()
    a, sa = _matrix(0, 256, 1, 1)
    w, sw = _matrix(16, 256, 128, 1)
    mb.mb_matmul_q8(a, sa, w, sw, torch.empty(0, 16, device=DEV))


@pytest.mark.parametrize("rows, n, width, dtype", [(131072, 8200, 32, "bf16"), (140000, 4096, 2304, "bf16"), (16, 65536, 16384, "f32")])
def test_offsets_beyond_32_bits(rows, n, width, dtype):
    a, sa = _matrix(rows, width, 1, 9)
    w, sw = _matrix(n, width, 128, 10)
    out = torch.empty(rows, n, dtype=TYPES[dtype], device=DEV)
    mb.mb_matmul_q8(a, sa, w, sw, out)
    r = torch.unique(torch.tensor([0, 1, rows // 2, rows - 2, rows - 1], device=DEV))
    block = (n - 1) // 128   # the last block of columns, and the first
    for c, b in ((slice(0, 128), 0), (slice(128 * block, n), block)):
        _check(a[r], sa[r], w[c], sw[b:b + 1], out[r][:, c], dtype)
