"""The training operators' native marshalling and plain path agree on arguments
that are given as None."""
import pytest
import torch

from paper_2401_13660_gb300 import mbscan as mb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("missing", [("dbias",), ("dstate",), ("dw",), ("dx",), ("dbias", "dstate"), ("dx", "dw", "dbias", "dstate")])
@pytest.mark.parametrize("explicit", [True, False])
def test_gradients_that_are_not_given_are_made(missing, explicit):
    g = torch.Generator(device=DEV).manual_seed(3)
    rnd = lambda *s: torch.randn(*s, device=DEV, generator=g)
    x, w, dout, bias, state = rnd(2, 9, 16), rnd(16, 4), rnd(2, 9, 16), rnd(16), rnd(2, 3, 16)
    want = mb.mb_conv1d_backward(x, w, dout, bias=bias, state=state, dstate_out=state)
    assert all(v is not None for v in want.values())
    ws = torch.zeros(mb.mb_conv1d_backward_workspace_size(2, 9, 16), dtype=torch.uint8, device=DEV)
    for kw in (dict(ws=ws), dict(), dict(ws=ws, stream=torch.cuda.current_stream())):
        grads = {k: torch.empty_like(v) for k, v in want.items() if k not in missing}
        if explicit:
            grads.update({k: None for k in missing})
        got = mb.mb_conv1d_backward(x, w, dout, bias=bias, state=state, dstate_out=state, grads=grads, **kw)
        assert set(got) == set(want) and all(torch.equal(got[k], v) for k, v in want.items())
        assert all(got[k] is grads[k] for k in grads if grads[k] is not None)
