"""CPU checks of the C ABI of 8-bit projections and sampling: bad arguments are refused on the host before any launch, so
these run without a GPU."""
import pytest
import torch

from paper_2401_13660_gb300 import mbscan as mb

BASE = 1 << 40   # aligned, never dereferenced stand-ins for device addresses
A, B, C, D, E, F, G, H = (BASE + i * (1 << 36) for i in range(8))
OK, BAD, UNSUPPORTED = mb.MB_OK, mb.MB_ERR_INVALID_ARG, mb.MB_ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def lib():
    return mb.load_library()


def test_scale_stride(lib):
    assert [lib.mb_q8_scale_stride(w) for w in (0, 16, 512, 528, 1024, 2304, -16, 24, 1 << 32)] == [0, 4, 4, 8, 8, 20, 0, 0, 0]


@pytest.mark.parametrize("change, want", [
    (dict(rows=-1), BAD), (dict(width=-16), BAD), (dict(width=40), UNSUPPORTED), (dict(rows=1 << 31, width=32), BAD),
    (dict(rows=(1 << 31) + 1), BAD), (dict(dtype=2), BAD), (dict(eps=-1.0), BAD), (dict(eps=float("nan")), BAD),
    (dict(residual=None), BAD), (dict(w=None), BAD), (dict(q=None), BAD), (dict(scales=None), BAD), (dict(add=A + 8), BAD),
    (dict(residual=B + 4), BAD), (dict(w=C + 8), BAD), (dict(q=D + 8), BAD), (dict(scales=E + 2), BAD),
    (dict(q=B + 4096), BAD), (dict(scales=D + 32), BAD), (dict(add=B), BAD), (dict(w=D), BAD), (dict(scales=C), BAD),
    (dict(rows=0), OK), (dict(width=0), OK)])
def test_rmsnorm(lib, change, want):
    a = dict(add=A, dtype=1, residual=B, w=C, eps=1e-5, q=D, scales=E, rows=4, width=1024) | change
    assert lib.mb_rmsnorm_q8(a["add"], a["dtype"], a["residual"], a["w"], a["eps"], a["q"], a["scales"], a["rows"], a["width"],
                             None) == want


@pytest.mark.parametrize("change, want", [
    (dict(rows=-1), BAD), (dict(width=24), UNSUPPORTED), (dict(rows=1 << 31, width=32), BAD), (dict(dtype=5), BAD),
    (dict(block_rows=0), BAD), (dict(block_rows=64), BAD), (dict(x_stride=1008), BAD), (dict(x_stride=1028), BAD),
    (dict(x_stride=-1), BAD), (dict(x_stride=1 << 32), BAD), (dict(x=None), BAD), (dict(q=None), BAD), (dict(scales=None), BAD),
    (dict(x=A + 8), BAD), (dict(q=B + 4), BAD), (dict(scales=C + 1), BAD), (dict(q=A), BAD), (dict(scales=A + 6000), BAD),
    (dict(q=A + 3 * 4096 + 2048 - 16, x_stride=2048), BAD), (dict(scales=B + 1024), BAD), (dict(rows=0), OK), (dict(width=0, x_stride=0), OK)])
def test_quantize(lib, change, want):
    a = dict(x=A, dtype=1, x_stride=0, block_rows=1, q=B, scales=C, rows=4, width=1024) | change
    assert lib.mb_quantize_q8(a["x"], a["dtype"], a["x_stride"], a["block_rows"], a["q"], a["scales"], a["rows"], a["width"],
                              None) == want


@pytest.mark.parametrize("change, want", [
    (dict(rows=-1), BAD), (dict(width=8), UNSUPPORTED), (dict(dtype=-1), BAD), (dict(block_rows=2), BAD), (dict(q=None), BAD),
    (dict(scales=None), BAD), (dict(out=None), BAD), (dict(out=C + 4), BAD), (dict(q=A + 8), BAD), (dict(scales=B + 2), BAD),
    (dict(out=A), BAD), (dict(out=B - 4096), BAD), (dict(rows=0), OK)])
def test_dequantize(lib, change, want):
    a = dict(q=A, scales=B, block_rows=128, out=C, dtype=0, rows=4, width=1024) | change
    assert lib.mb_dequantize_q8(a["q"], a["scales"], a["block_rows"], a["out"], a["dtype"], a["rows"], a["width"], None) == want


@pytest.mark.parametrize("change, want", [
    (dict(rows=-1), BAD), (dict(n_out=-8), BAD), (dict(width=-16), BAD), (dict(width=40), UNSUPPORTED), (dict(n_out=260), UNSUPPORTED),
    (dict(dtype=3), BAD), (dict(rows=1 << 28, n_out=16), BAD), (dict(rows=1 << 22, width=1024), BAD), (dict(n_out=1 << 28), BAD),
    (dict(part=64), BAD), (dict(part=384), BAD), (dict(part=-128), BAD), (dict(part=1024), BAD),
    (dict(a=None), BAD), (dict(a_scales=None), BAD), (dict(w=None), BAD), (dict(w_scales=None), BAD), (dict(out=None), BAD),
    (dict(a=A + 8), BAD), (dict(a_scales=B + 2), BAD), (dict(w=C + 4), BAD), (dict(w_scales=D + 1), BAD), (dict(out=E + 8), BAD),
    (dict(out=A), BAD), (dict(out=B), BAD), (dict(out=C), BAD), (dict(out=D), BAD), (dict(ws=F + 128), BAD),
    (dict(ws=F, ws_bytes=255), BAD), (dict(ws=E), BAD), (dict(ws=C), BAD), (dict(rows=0), OK), (dict(n_out=0), OK)])
def test_matmul(lib, change, want):
    a = dict(a=A, a_scales=B, w=C, w_scales=D, out=E, dtype=1, rows=32, n_out=512, width=1024, part=0, ws=None, ws_bytes=256) | change
    assert lib.mb_matmul_q8(a["a"], a["a_scales"], a["w"], a["w_scales"], a["out"], a["dtype"], a["rows"], a["n_out"], a["width"],
                            a["part"], a["ws"], a["ws_bytes"], None) == want


@pytest.mark.parametrize("change, want", [
    (dict(dtype=2), BAD), (dict(kind=0), BAD), (dict(kind=3), BAD), (dict(n=-1), BAD), (dict(vocab=0), BAD), (dict(vocab=-1), BAD),
    (dict(vocab=(1 << 30) + 1), BAD), (dict(n=1 << 24), BAD), (dict(logits=None), BAD), (dict(u=None), BAD), (dict(tokens=None), BAD),
    (dict(logits=A + 8), BAD), (dict(tokens=C + 4), BAD), (dict(u=B + 2), BAD), (dict(temperature=D + 1), BAD), (dict(top_k=E + 2), BAD),
    (dict(top_p=F + 3), BAD), (dict(min_p=G + 1), BAD), (dict(prob=H + 2), BAD), (dict(tokens=A + 1024), BAD), (dict(tokens=B), BAD),
    (dict(prob=C + 8), BAD), (dict(prob=A), BAD), (dict(tokens=E), BAD), (dict(prob=G), BAD), (dict(n=0), OK)])
def test_sample(lib, change, want):
    a = dict(logits=A, dtype=0, u=B, temperature=D, top_k=E, top_p=F, min_p=G, tokens=C, kind=2, prob=H, n=16, vocab=256) | change
    assert lib.mb_sample(a["logits"], a["dtype"], a["u"], a["temperature"], a["top_k"], a["top_p"], a["min_p"], a["tokens"], a["kind"],
                         a["prob"], a["n"], a["vocab"], None) == want


def test_the_binding_refuses_what_does_not_fit():
    """Shapes, types and host memory, before any launch."""
    q, s = torch.zeros(4, 256, dtype=torch.uint8), torch.zeros(4, 4, dtype=torch.uint8)
    x, w = torch.zeros(4, 256), torch.zeros(256)
    for bad in (dict(q=torch.zeros(4, 256, dtype=torch.int8)), dict(q=q[:3]), dict(scales=torch.zeros(4, 2, dtype=torch.uint8)),
                dict(w=w[:128]), dict(residual=x.double()), dict(add=x.half()), dict(add=x[:2]), dict()):
        a = dict(residual=x, w=w, q=q, scales=s, add=x) | bad
        with pytest.raises((TypeError, ValueError)):
            mb.mb_rmsnorm_q8(a["residual"], a["w"], a["q"], a["scales"], add=a["add"])
    for bad in (dict(x=x.half()), dict(x=x[:3]), dict(block_rows=2), dict(x=x.t()), dict(q=q.view(2, 512)), dict()):
        a = dict(x=x, q=q, scales=s, block_rows=1) | bad
        with pytest.raises((TypeError, ValueError)):
            mb.mb_quantize_q8(a["x"], a["q"], a["scales"], block_rows=a["block_rows"])
    wide = torch.zeros(4096)
    for strides in ((256, 2), (512, 2), (1, 4), (0, 1), (255, 1)):
        with pytest.raises(ValueError, match="column block"):
            mb.mb_quantize_q8(torch.as_strided(wide, (4, 256), strides), q, s)
    for bad in (dict(out=x.half()), dict(out=x[:3]), dict(block_rows=128), dict()):
        a = dict(out=x, block_rows=1) | bad
        with pytest.raises((TypeError, ValueError)):
            mb.mb_dequantize_q8(q, s, a["out"], block_rows=a["block_rows"])
    wq, ws = torch.zeros(256, 256, dtype=torch.uint8), torch.zeros(2, 4, dtype=torch.uint8)
    out = torch.zeros(4, 256)
    for bad in (dict(a=q.view(8, 128)), dict(w=wq[:, :128].contiguous()), dict(sw=ws[:1]), dict(out=out.half()), dict(out=out[:2]),
                dict(out=torch.zeros(3, 4, 128)), dict(out=torch.zeros(2, 5, 128)), dict(ws=torch.zeros(256)), dict()):
        a = dict(a=q, sa=s, w=wq, sw=ws, out=out, ws=None) | bad
        with pytest.raises((TypeError, ValueError)):
            mb.mb_matmul_q8(a["a"], a["sa"], a["w"], a["sw"], a["out"], ws=a["ws"])
    u, tok = torch.zeros(4), torch.zeros(4, dtype=torch.int64)
    for bad in (dict(logits=x.half()), dict(u=u[:3]), dict(u=None), dict(u=u.double()), dict(tokens=tok.byte()), dict(tokens=tok[:2]),
                dict(top_k=tok), dict(top_p=u.double()), dict(temperature=u[:1]), dict(min_p=tok), dict(prob=u.bfloat16()), dict()):
        a = dict(logits=x, u=u, tokens=tok, temperature=None, top_k=None, top_p=None, min_p=None, prob=None) | bad
        with pytest.raises((TypeError, ValueError)):
            mb.mb_sample(a["logits"], a["u"], a["tokens"], **{k: a[k] for k in ("temperature", "top_k", "top_p", "min_p", "prob")})
