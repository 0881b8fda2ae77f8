"""Host-side checks of the training operators' C entry points (CPU: no call here
reaches the device with anything but arguments that are refused, or fails to
launch without one)."""
import ctypes

import pytest

from paper_2401_13660_gb300 import mbscan as mb

FAKE = 1 << 40   # an aligned, never-dereferenced stand-in for a device address
RUN = (mb.MB_OK, mb.MB_ERR_CUDA)


def _at(i):
    return FAKE + (i << 34)


def _conv(**kw):
    a = mb.mb_conv1d_args(2, 8, 64, mb.MB_BF16, 0, _at(0), _at(1), _at(2), _at(3))
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.fixture(scope="module")
def lib():
    import torch
    if torch.cuda.is_available():
        pytest.skip("stand-in addresses: only where nothing can be launched")
    return mb.load_library()


def test_conv1d(lib):
    def call(a=None, out=_at(4), so=_at(5)):
        return lib.mb_conv1d(ctypes.byref(a or _conv()), out, so, None)
    assert call() in RUN and call(so=None) in RUN and call(so=_at(1)) in RUN
    assert call(_conv(x_stride=128)) in RUN and call(_conv(state=None, bias=None)) in RUN
    assert call(_conv(width=60)) == mb.MB_ERR_UNSUPPORTED
    for a in (_conv(dtype=5), _conv(batch=-1), _conv(seqlen=-1), _conv(width=-8), _conv(x_stride=56), _conv(x_stride=68),
              _conv(x=None), _conv(w=None), _conv(x=_at(0) + 8), _conv(bias=_at(3) + 4), _conv(seqlen=1 << 30),
              _conv(batch=1 << 40)):
        assert call(a) == mb.MB_ERR_INVALID_ARG
    for kw in (dict(out=None), dict(out=_at(4) + 2), dict(out=_at(0) + 64), dict(out=_at(1)), dict(out=_at(2)),
               dict(so=_at(0)), dict(so=_at(1) + 16), dict(so=_at(4) + 16), dict(so=_at(5) + 8)):
        assert call(**kw) == mb.MB_ERR_INVALID_ARG
    assert lib.mb_conv1d(None, _at(4), None, None) == mb.MB_ERR_INVALID_ARG
    assert call(_conv(batch=0)) == mb.MB_OK and call(_conv(seqlen=0, x=None), out=None, so=None) == mb.MB_OK


def test_conv1d_backward(lib):
    need = lib.mb_conv1d_backward_workspace_size(2, 8, 64)
    assert need > 256 and lib.mb_conv1d_backward_workspace_size(2, 8, 60) == 0
    assert lib.mb_conv1d_backward_workspace_size(0, 8, 64) == 256
    assert lib.mb_conv1d_backward_workspace_size(1 << 30, 8, 64) == 0

    def call(a=None, dout=_at(4), dso=_at(5), ws=_at(10), wb=need, **kw):
        g = mb.mb_conv1d_grads(_at(6), 0, _at(7), _at(8), _at(9))
        for k, v in kw.items():
            setattr(g, k, v)
        return lib.mb_conv1d_backward(ctypes.byref(a or _conv()), dout, dso, ctypes.byref(g), ws, wb, None)
    assert call() in RUN and call(dstate=None, dbias=None, dso=None) in RUN and call(dx_stride=128) in RUN
    for kw in (dict(dout=None), dict(dx=None), dict(dw=None), dict(dx=_at(0)), dict(dx=_at(4) + 16), dict(dw=_at(2)),
               dict(dbias=_at(8) + 16), dict(dstate=_at(5)), dict(dx_stride=60), dict(dx_stride=68), dict(ws=None),
               dict(wb=need - 1), dict(ws=_at(10) + 16), dict(ws=_at(6)), dict(dw=_at(8) + 4)):
        assert call(**kw) == mb.MB_ERR_INVALID_ARG, kw
    assert call(_conv(width=0)) == mb.MB_OK


def test_embed(lib):
    def call(tok=_at(0), tt=0, table=_at(1), td=mb.MB_BF16, out=_at(2), od=mb.MB_F32, n=10, vocab=256, width=64):
        return lib.mb_embed(tok, tt, table, td, 1.0, out, od, n, vocab, width, None)
    assert call() in RUN and call(tt=2) in RUN and call(tok=_at(0) + 1) in RUN
    assert call(width=60) == mb.MB_ERR_UNSUPPORTED and call(width=1 << 21) == mb.MB_ERR_UNSUPPORTED
    for kw in (dict(tt=3), dict(td=2), dict(od=-1), dict(n=-1), dict(vocab=-1), dict(n=1 << 26), dict(vocab=1 << 26),
               dict(tok=None), dict(table=None), dict(out=None), dict(tok=_at(0) + 2, tt=1), dict(table=_at(1) + 8),
               dict(out=_at(2) + 4), dict(out=_at(1) + 64), dict(out=_at(0))):
        assert call(**kw) == mb.MB_ERR_INVALID_ARG, kw
    assert call(n=0, tok=None, out=None) == mb.MB_OK and call(vocab=0, table=None) in RUN


def test_embed_backward(lib):
    need = lib.mb_embed_backward_workspace_size(10, 256, 64)
    assert need > 256 and lib.mb_embed_backward_workspace_size(10, 256, 60) == 0

    def call(tok=_at(0), tt=0, dout=_at(1), dt=mb.MB_F32, d=_at(2), n=10, vocab=256, width=64, ws=_at(3), wb=need):
        return lib.mb_embed_backward(tok, tt, dout, dt, 1.0, 0, d, n, vocab, width, ws, wb, None)
    assert call() in RUN and call(n=0, tok=None, dout=None) in RUN
    for kw in (dict(tt=-1), dict(dt=9), dict(n=-1), dict(tok=None), dict(dout=None), dict(d=None), dict(d=_at(2) + 4),
               dict(d=_at(1)), dict(ws=None), dict(ws=_at(3) + 16), dict(wb=need - 1), dict(ws=_at(2)), dict(ws=_at(1)),
               dict(tok=_at(0) + 4, tt=2)):
        assert call(**kw) == mb.MB_ERR_INVALID_ARG, kw
    assert call(vocab=0) == mb.MB_OK and call(width=0) == mb.MB_OK


def test_cross_entropy(lib):
    def call(l=_at(0), dt=mb.MB_BF16, tgt=_at(1), tt=2, w=_at(2), loss=_at(3), d=_at(4), n=10, vocab=257):
        return lib.mb_cross_entropy(l, dt, tgt, tt, w, 1.0, loss, d, n, vocab, None)
    assert call() in RUN and call(w=None, d=None) in RUN and call(d=_at(0)) in RUN
    for kw in (dict(dt=4), dict(tt=4), dict(n=-1), dict(vocab=0), dict(n=1 << 30), dict(l=None), dict(tgt=None), dict(loss=None),
               dict(l=_at(0) + 2), dict(d=_at(0) + 16), dict(loss=_at(0)), dict(loss=_at(4)), dict(loss=_at(2)),
               dict(tgt=_at(1) + 4), dict(w=_at(2) + 2), dict(d=_at(1))):
        assert call(**kw) == mb.MB_ERR_INVALID_ARG, kw
    assert call(n=0, l=None, tgt=None, loss=None) == mb.MB_OK


def test_grad_norm_and_clip(lib):
    def lst(*entries):
        return (mb.mb_tensor * len(entries))(*(mb.mb_tensor(*e) for e in entries))
    ok = lst((_at(0), 10, mb.MB_F32, 0), (_at(1) + 2, 7, mb.MB_BF16, 0), (None, 0, mb.MB_F32, 0))
    need = lib.mb_grad_norm_workspace_size()

    def norm(l=ok, n=3, out=_at(5), ws=_at(6), wb=need):
        return lib.mb_grad_norm(l, n, out, ws, wb, None)
    assert norm() in RUN and norm(l=None, n=0) in RUN
    bad = [lst((_at(0), -1, 0, 0)), lst((None, 1, 0, 0)), lst((_at(0) + 2, 4, 0, 0)), lst((_at(0), 4, 3, 0)),
           lst((_at(0), 1 << 50, 0, 0)), lst((_at(0), 4, 0, 1)), lst((_at(5) - 16, 8, 0, 0)), lst((_at(6), 8, 0, 0))]
    for l in bad:
        assert norm(l=l, n=1) == mb.MB_ERR_INVALID_ARG
    for kw in (dict(l=None), dict(n=-1), dict(out=None), dict(out=_at(5) + 2), dict(ws=None), dict(ws=_at(6) + 64),
               dict(wb=need - 8), dict(out=_at(6))):
        assert norm(**kw) == mb.MB_ERR_INVALID_ARG, kw

    def clip(l=ok, out=None, n=3, nrm=_at(5), most=1.0):
        return lib.mb_grad_clip(l, out, n, nrm, most, None)
    assert clip() in RUN and clip(out=ok) in RUN
    assert clip(out=lst((_at(8), 10, mb.MB_BF16, 0), (_at(9), 7, mb.MB_F32, 0), (None, 0, 0, 0))) in RUN
    for kw in (dict(nrm=None), dict(most=0.0), dict(most=-1.0), dict(most=float("nan")), dict(l=bad[0], n=1),
               dict(out=lst((_at(8), 9, 0, 0)), n=1), dict(out=lst((_at(0) + 4, 10, 0, 0)), n=1),
               dict(out=lst((_at(0), 10, mb.MB_BF16, 0)), n=1), dict(nrm=_at(0) + 8)):
        assert clip(**kw) == mb.MB_ERR_INVALID_ARG, kw
