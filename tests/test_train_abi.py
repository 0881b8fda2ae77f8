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
