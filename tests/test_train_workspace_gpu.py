"""The training operators write nothing behind a workspace of exactly the size
they ask for, whatever lies in it before (but the cleared status block)."""
import pytest
import torch

from paper_2401_13660_gb300 import mbscan as mb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BEHIND = 1 << 16


def _exact(need):
    """A workspace of `need` bytes of ones with more of them behind it."""
    buffer = torch.full((need + BEHIND,), 255, dtype=torch.uint8, device=DEV)
    buffer[:256] = 0
    return buffer, buffer[:need]


def _untouched(buffer, need):
    return bool((buffer[need:] == 255).all()) and not buffer[:256].any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n, vocab, width", [(1, 1, 8), (1, 300, 8), (2, 256, 16), (17, 5, 32), (63, 256, 8), (64, 70000, 8), (65, 3, 16),
                                             (1025, 1, 8), (300, 5, 1040), (8200, 256, 2304), (140000, 256, 8)])
def test_table_gradient(n, vocab, width, dtype):
    g = torch.Generator(device=DEV).manual_seed(n + width)
    tok = torch.randint(-1, vocab, (n,), device=DEV, generator=g)
    dout = torch.randint(-8, 9, (n, width), device=DEV, generator=g).to(dtype)   # whole numbers: exact in any order
    need = mb.mb_embed_backward_workspace_size(n, vocab, width)
    buffer, ws = _exact(need)
    d = torch.full((vocab, width), 7.0, device=DEV)
    mb.mb_embed_backward(tok, dout, d, ws=ws)
    want = torch.zeros(vocab, width, device=DEV, dtype=torch.float64)
    want.index_add_(0, tok[tok >= 0], dout[tok >= 0].double())
    assert torch.equal(d.double(), want) and _untouched(buffer, need)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("batch, L, width", [(1, 1, 8), (3, 0, 16), (1, 2, 264), (2, 65, 72), (33, 16, 128), (1, 3000, 1544)])
def test_convolution(batch, L, width, dtype):
    g = torch.Generator(device=DEV).manual_seed(L + width)
    rnd = lambda *s: torch.randn(*s, device=DEV, generator=g)
    x, dout, w, bias = rnd(batch, L, width).to(dtype), rnd(batch, L, width).to(dtype), rnd(width, 4), rnd(width)
    need = mb.mb_conv1d_backward_workspace_size(batch, L, width)
    buffer, ws = _exact(need)
    got = mb.mb_conv1d_backward(x, w, dout, bias=bias, ws=ws)
    want = mb.mb_conv1d_backward(x, w, dout, bias=bias)
    assert all(torch.equal(got[k], want[k]) for k in ("dx", "dw", "dbias")) and _untouched(buffer, need)


@pytest.mark.parametrize("sizes", [[1], [5000, 3], [100003] * 40, [7] * 2000])
def test_norm(sizes):
    need = mb.mb_grad_norm_workspace_size()
    buffer, ws = _exact(need)
    norm = mb.mb_grad_norm([torch.full((n,), 2.0, device=DEV) for n in sizes], ws=ws)
    assert abs(float(norm) - 2 * sum(sizes) ** 0.5) <= 1e-5 * float(norm) and _untouched(buffer, need)
