"""mb_dequantize_q8 at the ends of the scales: exact down to 2^-136, what 2^-127 makes of e4m3's least number, and infinite
beyond the type's range."""
import numpy as np
import pytest
import torch

from oracle import serve
from paper_2401_13660_gb300 import mbscan as mb

from _parity import to_np

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("scale", [0, 1, 2, 8, 126, 127, 246, 247, 253, 254])
def test_ends(scale, dtype):
    q = torch.arange(256, dtype=torch.uint8, device=DEV).view(1, 256)
    s = torch.full((1, 4), scale, dtype=torch.uint8, device=DEV)
    out = mb.mb_dequantize_q8(q, s, torch.empty(1, 256, dtype=dtype, device=DEV))
    exact = serve.dequantize(q.cpu().numpy(), s.cpu().numpy(), 1)
    with np.errstate(over="ignore"):
        want = torch.tensor(exact).to(dtype)
    assert torch.equal(out.cpu().isnan(), want.isnan()) and torch.equal(out.cpu().nan_to_num(7, 1e30, -1e30), want.nan_to_num(7, 1e30, -1e30))
    if dtype == torch.float32:
        got = to_np(out)
        assert np.array_equal(got[np.isfinite(got)], exact[np.isfinite(got)])   # no rounding at all
