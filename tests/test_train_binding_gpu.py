"""The native argument marshalling of the training operators against the plain
Python path, which a `stream` argument selects: the same results bit for bit,
and wrong arguments left to the plain path, which raises."""
import pytest
import torch

from paper_2401_13660_gb300 import mbscan as mb

from test_native_binding_gpu import _spy

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("full", [True, False])
@pytest.mark.parametrize("b, L, D", [(2, 5, 16), (1, 1, 64), (3, 1, 24)])
def test_native_equals_plain(monkeypatch, full, b, L, D):
    served = _spy(monkeypatch)
    ty = torch.bfloat16 if full else torch.float32
    g = torch.Generator(device=DEV).manual_seed(b + L + D)
    rnd = lambda *s, dtype=torch.float32: torch.randn(*s, device=DEV, generator=g).to(dtype)
    x = rnd(b, L, 2 * D, dtype=ty)[..., :D]
    w, bias, state = rnd(D, 4), rnd(D) if full else None, rnd(b, 3, D, dtype=ty) if full else None
    dout, table = rnd(b, L, D, dtype=ty), rnd(256, D, dtype=ty)
    tokens = torch.randint(0, 256, (b, L), device=DEV, generator=g).to(torch.uint8 if full else torch.int64)
    logits, weight = rnd(b, L, 256, dtype=ty), torch.rand(b, L, device=DEV, generator=g) if full else None
    grads = [rnd(100), rnd(33, dtype=ty)]

    def every(stream):
        n = dict(stream=stream)
        new = lambda *s, dtype=torch.float32: torch.zeros(*s, device=DEV, dtype=dtype)
        ws = new(1 << 20, dtype=torch.uint8)
        out = [mb.mb_conv1d(x, w, new(b, L, D, dtype=ty), bias=bias, state=state, state_out=new(b, 3, D, dtype=ty), **n)]
        gr = dict(dx=new(b, L, 3 * D, dtype=ty)[..., :D], dw=new(D, 4))
        if full:
            gr.update(dbias=new(D), dstate=new(b, 3, D, dtype=ty))
        got = mb.mb_conv1d_backward(x, w, dout, bias=bias, state=state, dstate_out=state, grads=gr, ws=ws, **n)
        out += [got[k] for k in ("dx", "dw", "dbias", "dstate")]
        out.append(mb.mb_embed(tokens, table, new(b, L, D), scale=1.5, **n))
        out.append(mb.mb_embed_backward(tokens, dout, new(256, D), scale=1.5, accumulate=full, ws=ws, **n))
        out += mb.mb_cross_entropy(logits, tokens, new(b, L), torch.zeros_like(logits) if full else None, weight=weight,
                                   scale=0.25, **n)
        ts = [t.clone() for t in grads]
        lst = mb.mb_tensor_list(ts)
        norm = mb.mb_grad_norm(lst, new(1), ws=ws, **n)
        o = None if full else [torch.zeros_like(t, dtype=torch.float32) for t in ts]
        mb.mb_grad_clip(lst, norm, 0.5, out=None if full else mb.mb_tensor_list(o), **n)
        return out + [norm] + (ts if full else o)
    native = every(None)
    assert set(served) == {"conv1d", "conv1d_backward", "embed", "embed_backward", "cross_entropy", "grad_norm", "grad_clip"}
    torch.cuda.synchronize()
    for p, q in zip(native, every(torch.cuda.current_stream())):
        assert (p is None and q is None) or torch.equal(p, q)


def test_wrong_arguments_are_left_to_the_plain_path(monkeypatch):
    served = _spy(monkeypatch)
    t = lambda *s, dtype=torch.float32: torch.zeros(*s, device=DEV, dtype=dtype)
    ws = t(1 << 16, dtype=torch.uint8)
    bad = [lambda: mb.mb_conv1d(t(1, 2, 8), t(8, 4), t(1, 2, 16)), lambda: mb.mb_conv1d(t(1, 2, 8), t(8, 4, dtype=torch.float64), t(1, 2, 8)),
           lambda: mb.mb_conv1d_backward(t(1, 2, 8), t(8, 4), t(1, 2, 8), grads=dict(dx=t(1, 2, 8).cpu(), dw=t(8, 4)), ws=ws),
           lambda: mb.mb_embed(t(3), t(4, 8), t(3, 8)), lambda: mb.mb_embed(t(3, dtype=torch.uint8), t(4, 8), t(3, 16)),
           lambda: mb.mb_embed_backward(t(3, dtype=torch.uint8), t(2, 8), t(4, 8), ws=ws),
           lambda: mb.mb_cross_entropy(t(3, 8), t(3, dtype=torch.int16), t(3)), lambda: mb.mb_cross_entropy(t(3, 8), t(3, dtype=torch.uint8), t(4)),
           lambda: mb.mb_grad_norm(mb.mb_tensor_list([t(3)]), t(2), ws=ws),
           lambda: mb.mb_grad_clip(mb.mb_tensor_list([t(3)]), t(1).cpu(), 1.0),
           lambda: mb.mb_grad_clip(mb.mb_tensor_list([t(3)]), t(1), 1.0, out=mb.mb_tensor_list([t(3), t(3)]))]
    for f in bad:
        with pytest.raises((TypeError, ValueError)):
            f()
    assert not served
