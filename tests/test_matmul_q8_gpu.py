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
