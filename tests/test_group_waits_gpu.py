"""A group of warps whose waits have limits of their own gives up together: the diagnostic makes one of four warps give up
and lets the others see the phase that it waited for complete."""
import pytest
import torch

from paper_2401_13660_gb300 import mbscan as mb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("limit", [1, 1000, 100_000, 10_000_000])
def test_all_give_up_with_the_first(limit):
    ws = torch.zeros(256, dtype=torch.uint8, device=DEV)
    for _ in range(3):
        mb.mb_selftest_timeout(ws, limit)
        st, detail = mb.mb_check(ws)
        assert st == mb.MB_ERR_TIMEOUT and detail > limit


def test_products_go_on_after_it():
    """The same status block, then a product of several tiles to a CTA: sums are moved by groups that wait as one."""
    ws = torch.zeros(256, dtype=torch.uint8, device=DEV)
    mb.mb_selftest_timeout(ws, 100_000)
    assert mb.mb_check(ws)[0] == mb.MB_ERR_TIMEOUT
    a, w = (torch.ones(n, 256, device=DEV).to(torch.float8_e4m3fn) for n in (40000, 128))
    sa, sw = (torch.full((n, 4), 127, dtype=torch.uint8, device=DEV) for n in (40000, 1))
    for dtype in (torch.bfloat16, torch.float32):
        out = torch.empty(40000, 128, dtype=dtype, device=DEV)
        mb.mb_matmul_q8(a, sa, w, sw, out, ws=ws)
        assert (out == 256).all()
    assert mb.mb_check(ws) == (mb.MB_OK, -1)
