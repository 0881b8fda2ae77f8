"""Rounding to 8 bits with block scales (mb_quantize_q8, mb_rmsnorm_q8, mb_dequantize_q8) against the definition in 64 bits
(oracle/serve.py).

What is given is rounded exactly: scaling by a power of two is exact in fp32 (what it pushes below the subnormals is 0 in
e4m3 either way), so bytes and scales are those of the definition. The norm carries its rounding errors along, to about 2^-44,
and rounds once: its values, too, are those of the definition, but for a value in 2^40 of those near a border."""
import numpy as np
import pytest
import torch

from oracle import serve
from paper_2401_13660_gb300 import mbscan as mb

from _parity import to_np

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZES = [(1, 16), (1, 128), (3, 144), (2, 512), (5, 528), (127, 256), (129, 640), (300, 64), (7, 2304), (2, 20496)]


def _empty(rows, width, block_rows):
    q = torch.full((rows, width), 0x55, dtype=torch.uint8, device=DEV)
    s = torch.full((-(-rows // block_rows), serve.stride(width)), 0x55, dtype=torch.uint8, device=DEV)
    return q, s


def _values(rows, width, dtype, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed + rows + width)
    x = torch.randn(rows, width, device=DEV, generator=g) * torch.exp(3 * torch.randn(rows, 1, device=DEV, generator=g))
    return x.to(TYPES[dtype])


def _check(x, q, s, block_rows):
    rq, rs = serve.quantize(to_np(x), block_rows)
    got = serve.e4m3_values(q.cpu().numpy())
    assert np.array_equal(s.cpu().numpy(), rs)
    assert np.array_equal(got, rq, equal_nan=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("rows, width", SIZES)
def test_quantize(rows, width, block_rows, dtype):
    x = _values(rows, width, dtype)
    q, s = _empty(rows, width, block_rows)
    mb.mb_quantize_q8(x, q.view(torch.float8_e4m3fn), s, block_rows=block_rows)
    _check(x, q, s, block_rows)


@pytest.mark.parametrize("block_rows", [1, 128])
def test_every_border(block_rows):
    """Halfway values of every spacing, the largest value at and around the scale's borders, the ends of fp32."""
    rows = []
    for top in (448.0, 448.0 * (1 + 2.0 ** -23), 224.0, 224.0 * (1 + 2.0 ** -23), 2.0 ** -149, 2.0 ** -126, 1.5 * 2.0 ** 127,
                float(np.finfo(np.float32).max), 1e-40, 0.0):
        v = np.zeros(128)
        v[0] = top
        grid = top * 2.0 ** -8 * np.linspace(-1.0, 1.0, 41)   # coarse, and what rounds at the bottom
        v[1:42] = np.float32(grid)
        v[42:42 + 64] = np.float32(np.arange(64) * top * 2.0 ** -18)
        rows.append(v)
    half = np.zeros(128)
    half[0] = 448.0
    half[1:] = [(8 + m + 0.5) * 2.0 ** (e - 3) for e in range(-6, 8) for m in range(8)][:64] + \
        [(m + 0.5) * 2.0 ** -9 for m in range(8)] * 7 + [2.0 ** -10, -2.0 ** -10, 2.0 ** -11, -0.0, 447.9, 432.0, 431.9]
    rows.append(half)
    x = torch.tensor(np.array(rows), dtype=torch.float32, device=DEV)
    if block_rows == 128:
        for i in range(len(rows)):
            q, s = _empty(1, 128, 128)
            mb.mb_quantize_q8(x[i:i + 1], q, s, block_rows=128)
            _check(x[i:i + 1], q, s, 128)
    else:
        q, s = _empty(len(rows), 128, 1)
        mb.mb_quantize_q8(x, q, s)
        _check(x, q, s, 1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_what_is_not_finite_stays_in_its_place(block_rows, dtype):
    x = _values(130, 400, dtype)
    x[3, 5], x[129, 399], x[0, 130:200], x[7] = float("nan"), float("inf"), -float("inf"), float("nan")
    q, s = _empty(130, 400, block_rows)
    mb.mb_quantize_q8(x, q, s, block_rows=block_rows)
    _check(x, q, s, block_rows)
    out = torch.empty(130, 400, device=DEV)
    mb.mb_dequantize_q8(q, s, out, block_rows=block_rows)
    assert torch.equal(out.isnan(), ~x.isfinite())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_column_block_of_wider_rows(dtype):
    wide = _values(33, 800, dtype)
    for x in (wide[:, 400:672], wide[:1, 16:32]):
        q, s = _empty(*x.shape, 1)
        mb.mb_quantize_q8(x, q, s)
        _check(x, q, s, 1)
        q, s = _empty(*x.shape, 128)
        mb.mb_quantize_q8(x, q, s, block_rows=128)
        _check(x, q, s, 128)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("rows, width", [(1, 16), (3, 144), (257, 1040)])
def test_dequantize_every_byte(rows, width, block_rows, dtype):
    g = torch.Generator(device=DEV).manual_seed(rows)
    q = torch.randint(0, 256, (rows, width), device=DEV, generator=g, dtype=torch.uint8)
    s = torch.randint(60, 200, (-(-rows // block_rows), serve.stride(width)), device=DEV, generator=g, dtype=torch.uint8)
    s[0, 0] = 0   # 2^-127
    if s.shape[0] > 1:
        s[1, 0] = 255
    out = torch.empty(rows, width, dtype=TYPES[dtype], device=DEV)
    mb.mb_dequantize_q8(q, s, out, block_rows=block_rows)
    want = torch.tensor(serve.dequantize(q.cpu().numpy(), s.cpu().numpy(), block_rows)).to(TYPES[dtype])
    got = out.cpu()
    assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(), want.nan_to_num())


@pytest.mark.parametrize("add", ["f32", "bf16", None])
@pytest.mark.parametrize("rows, width", SIZES + [(1300, 1024), (700, 2304), (620, 20000), (1, 32784)])
def test_rmsnorm(rows, width, add):
    g = torch.Generator(device=DEV).manual_seed(rows + width)
    residual = torch.randn(rows, width, device=DEV, generator=g)
    w = torch.rand(width, device=DEV, generator=g) + 0.5
    d = None if add is None else torch.randn(rows, width, device=DEV, generator=g).to(TYPES[add])
    want = residual if d is None else residual + d.float()
    q, s = _empty(rows, width, 1)
    mb.mb_rmsnorm_q8(residual, w, q, s, add=d, eps=1e-5)
    assert torch.equal(residual, want)
    q2, s2 = _empty(rows, width, 1)
    mb.mb_rmsnorm_q8(want, w, q2, s2)
    assert torch.equal(q, q2) and torch.equal(s, s2)
    some = slice(None) if rows <= 300 else slice(0, None, 97)
    rq, rs = serve.quantize(serve.rmsnorm(to_np(residual)[some], to_np(w), float(np.float32(1e-5))), 1)
    assert np.array_equal(s.cpu().numpy()[some], rs)
    assert np.array_equal(serve.e4m3_values(q.cpu().numpy()[some]), rq)


def test_rows_that_are_not_numbers():
    residual = torch.randn(4, 256, device=DEV)
    residual[1, 7], residual[2] = float("nan"), 0.0
    w = torch.ones(256, device=DEV)
    q, s = _empty(4, 256, 1)
    mb.mb_rmsnorm_q8(residual, w, q, s)
    v = serve.dequantize(q.cpu().numpy(), s.cpu().numpy(), 1)
    assert np.isnan(v[1]).all() and not v[2].any() and np.isfinite(v[[0, 2, 3]]).all()


def test_nothing_to_do():
    for rows, width in ((0, 256), (5, 0)):
        q, s = torch.empty(rows, width, dtype=torch.uint8, device=DEV), torch.empty(rows, serve.stride(width), dtype=torch.uint8, device=DEV)
        mb.mb_quantize_q8(torch.empty(rows, width, device=DEV), q, s)
        mb.mb_dequantize_q8(q, s, torch.empty(rows, width, device=DEV))
        mb.mb_rmsnorm_q8(torch.empty(rows, width, device=DEV), torch.empty(width, device=DEV), q, s)


def test_offsets_beyond_32_bits():
    rows, width = 131072, 16384   # 2^31 elements
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.randn(1024, width, device=DEV, generator=g, dtype=torch.bfloat16).repeat(rows // 1024, 1)
    x[-1] *= 3
    some = [0, 1, 65535, 65536, rows - 1]
    q = torch.empty(rows, width, dtype=torch.uint8, device=DEV)
    for block_rows in (1, 128):
        s = torch.empty(-(-rows // block_rows), serve.stride(width), dtype=torch.uint8, device=DEV)
        mb.mb_quantize_q8(x, q, s, block_rows=block_rows)
        last = slice(rows - 128, rows)
        if block_rows == 1:
            _check(x[some], q[some], s[some], 1)
        _check(x[last], q[last], s[-(128 // block_rows):], block_rows)
    out = torch.empty(rows, width, dtype=torch.bfloat16, device=DEV)
    mb.mb_dequantize_q8(q, s, out, block_rows=128)
    want = serve.dequantize(q[last].cpu().numpy(), s[-1:].cpu().numpy(), 128)
    assert np.array_equal(to_np(out[last]), want)
    del out, x
    residual = torch.randn(1024, width, device=DEV, generator=g).repeat(rows // 1024, 1)
    w = torch.rand(width, device=DEV, generator=g) + 0.5
    s = torch.empty(rows, serve.stride(width), dtype=torch.uint8, device=DEV)
    mb.mb_rmsnorm_q8(residual, w, q, s)
    rq, rs = serve.quantize(serve.rmsnorm(to_np(residual[some]), to_np(w), float(np.float32(1e-5))), 1)
    assert np.array_equal(serve.e4m3_values(q[some].cpu().numpy()), rq) and np.array_equal(s[some].cpu().numpy(), rs)


@pytest.mark.parametrize("scale", [1e-38, 1e-30, 1e-16, 1e15, 1e18, 1e37])
def test_norm_of_small_and_large_rows(scale):
    residual = torch.randn(7, 640, device=DEV) * scale
    w = torch.randn(640, device=DEV)
    w[3] = 1e30
    w[200:] *= 1e-20
    q, s = _empty(7, 640, 1)
    mb.mb_rmsnorm_q8(residual, w, q, s, eps=1e-5)
    rq, rs = serve.quantize(serve.rmsnorm(to_np(residual), to_np(w), float(np.float32(1e-5))), 1)
    got = serve.e4m3_values(q.cpu().numpy())
    # what is subnormal in fp32 on the way has fewer bits
    tiny = np.abs(serve.rmsnorm(to_np(residual), to_np(w), 1e-5)) < 2.0 ** -100
    assert np.array_equal(np.where(tiny, 0, got), np.where(tiny, 0, rq))


@pytest.mark.parametrize("width", [640, 20496])
@pytest.mark.parametrize("scale", [1e-37, 1e-25, 1.0])
def test_norm_without_eps(scale, width):
    residual = torch.randn(5, width, device=DEV) * scale
    w = torch.rand(width, device=DEV) + 0.5
    q, s = _empty(5, width, 1)
    mb.mb_rmsnorm_q8(residual, w, q, s, eps=0.0)
    rq, rs = serve.quantize(serve.rmsnorm(to_np(residual), to_np(w), 0.0), 1)
    assert np.array_equal(serve.e4m3_values(q.cpu().numpy()), rq) and np.array_equal(s.cpu().numpy(), rs)
