"""mb_grad_norm and mb_grad_clip against the 64-bit form (oracle/train.py).

Bounds, u = 2^-24: a sum of squares goes through fp32 chains of at most a few
hundred terms here (512 threads on units of 4096 elements) before 64 bits take
over: the norm is within 256 u. A clipped element is g times the fp32 quotient
max_norm / norm: within 3 u, plus half an ulp (2^-9) when it is bf16."""
import numpy as np
import pytest
import torch

from oracle import train
from paper_2401_13660_gb300 import mbscan as mb

from _parity import to_np

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
BF, F = torch.bfloat16, torch.float32


def _list(sizes, dtypes, seed=0, scale=1.0, offset=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    out = []
    for k, n in enumerate(sizes):
        t = (scale * torch.randn(n + offset, device=DEV, generator=g)).to(dtypes[k % len(dtypes)])
        out.append(t[offset:])
    return out


def _close(got, want, rel):
    return abs(got - want) <= rel * abs(want)


SIZES = [[1], [7], [8], [4096], [4097, 3], [1, 2, 3, 4, 5, 6, 7, 8, 9], [0, 5, 0], [100003, 64, 1, 8191], [2000000, 12345],
         [17] * 99, [33] * 100, [9] * 101, [2048] * 959, [31] * 960, [5] * 961, [1000] * 2500]


@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{s[0]}")
@pytest.mark.parametrize("dtypes", [(F,), (BF,), (BF, F, F)])
@pytest.mark.parametrize("offset", [0, 1, 3])
def test_norm_and_clip(sizes, dtypes, offset):
    ts = _list(sizes, dtypes, offset=offset)
    want = train.grad_norm([to_np(t) for t in ts])
    lst = mb.mb_tensor_list(ts)
    ws = torch.full((mb.mb_grad_norm_workspace_size(),), 255, dtype=torch.uint8, device=DEV)
    ws[:256] = 0
    norm = mb.mb_grad_norm(lst, ws=ws)
    assert _close(float(norm), want, 256 * U) and not ws[:256].any()
    assert torch.equal(norm, mb.mb_grad_norm(ts))     # reproducible, from the tensors themselves
    max_norm = 0.37 * want
    c = float(np.float32(max_norm)) / float(norm)
    for out_types in ((F,), (BF,), tuple(t.dtype for t in ts) or (F,)):
        out = [torch.full((t.numel() + offset,), 7.0, device=DEV, dtype=out_types[k % len(out_types)])[offset:]
               for k, t in enumerate(ts)]
        mb.mb_grad_clip(lst, norm, max_norm, out=out)
        for t, o in zip(ts, out):
            ref = to_np(t) * c
            bound = 2 * (3 * U + (2.0 ** -9 if o.dtype == BF else 0)) * np.abs(ref)
            assert np.all(np.abs(to_np(o) - ref) <= bound)
    keep = [t.clone() for t in ts]
    assert mb.mb_grad_clip(lst, norm, 2 * want) is lst            # below: nothing happens
    assert all(torch.equal(a, b) for a, b in zip(ts, keep))
    copy = [torch.empty_like(t) for t in ts]
    mb.mb_grad_clip(lst, norm, 2 * want, out=copy)                # or is copied
    assert all(torch.equal(a, b) for a, b in zip(copy, keep))
    mb.mb_grad_clip(lst, norm, max_norm)                          # in place: as into tensors of the same types
    assert all(torch.equal(a, b) for a, b in zip(ts, out))
    assert _close(float(mb.mb_grad_norm(lst)), max_norm, 2.0 ** -8 if BF in dtypes else 600 * U)


@pytest.mark.parametrize("scale", [1e-37, 1e-30, 1e-16, 1e-14, 1e14, 1e16, 1e30, 1e37])
@pytest.mark.parametrize("offset", [0, 1])
def test_squares_outside_the_fp32_range(scale, offset):
    ts = _list([50000, 77, 8], (F, BF), scale=scale, offset=offset) + _list([10], (F,), scale=1e-3 * scale)
    want = train.grad_norm([to_np(t) for t in ts])
    norm = mb.mb_grad_norm(ts)
    if want > 3e38:
        assert float(norm) == float("inf")
        return
    assert _close(float(norm), want, 512 * U)
    c = float(np.float32(want / 16)) / float(norm)
    ref = [to_np(t) * c for t in ts]
    mb.mb_grad_clip(ts, norm, want / 16)
    for t, r in zip(ts, ref):
        assert np.all(np.abs(to_np(t) - r) <= 2 * (3 * U + 2.0 ** -9) * np.abs(r) + 1e-40)


def test_mixed_magnitudes():
    ts = [torch.full((1000,), 1e-20, device=DEV), torch.full((1000,), 1.0, device=DEV), torch.full((1000,), 1e20, device=DEV)]
    assert _close(float(mb.mb_grad_norm(ts)), 1e20 * 1000 ** 0.5, 64 * U)
    assert _close(float(mb.mb_grad_norm(ts[:2])), 1000 ** 0.5, 64 * U)
    assert float(mb.mb_grad_norm([torch.zeros(5000, device=DEV)])) == 0.0


@pytest.mark.parametrize("dtype", [F, BF])
@pytest.mark.parametrize("at", [0, 4095, 9999])
def test_not_finite(dtype, at):
    for bad, is_bad in ((float("inf"), torch.isinf), (float("nan"), torch.isnan), (-float("inf"), torch.isinf)):
        t = torch.ones(10000, device=DEV, dtype=dtype)
        t[at] = bad
        rest = torch.ones(3000, device=DEV)
        norm = mb.mb_grad_norm([t, rest])
        assert is_bad(norm).all()
        keep = t.clone()
        mb.mb_grad_clip([t, rest], norm, 1.0)     # left as they are
        assert torch.equal(t.view(torch.uint8), keep.view(torch.uint8)) and (rest == 1).all()


def test_empty_lists_streams_and_graphs():
    norm = torch.full((1,), 9.0, device=DEV)
    assert float(mb.mb_grad_norm([], norm)) == 0.0
    mb.mb_grad_clip([], norm, 1.0)
    ts = _list([5000, 300, 7], (F, BF))
    want = mb.mb_grad_norm(ts)
    lst, ws = mb.mb_tensor_list(ts), torch.zeros(mb.mb_grad_norm_workspace_size(), dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    s = torch.cuda.Stream(DEV)
    mb.mb_grad_norm(lst, norm, ws=ws, stream=s)
    s.synchronize()
    assert torch.equal(norm, want)
    norm.zero_()
    out = [torch.empty(t.shape, device=DEV) for t in ts]
    olst = mb.mb_tensor_list(out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mb.mb_grad_norm(lst, norm, ws=ws)
        mb.mb_grad_clip(lst, norm, 1.0, out=olst)
    for t in ts:
        t.mul_(2)
    graph.replay()
    assert _close(float(norm), 2 * float(want), 4 * U)
    assert _close(float(mb.mb_grad_norm(out)), 1.0, 600 * U)


def test_more_elements_than_32_bits():
    n = (1 << 32) + 4099
    t = torch.zeros(n, device=DEV, dtype=BF)
    t[-1], t[1 << 31], t[0] = 2.0, 3.0, 6.0
    norm = mb.mb_grad_norm([t])
    assert float(norm) == 7.0
    mb.mb_grad_clip([t], norm, 3.5)
    assert t[-1] == 1.0 and t[1 << 31] == 1.5 and t[0] == 3.0


def test_refusals():
    t = torch.ones(100, device=DEV)
    n = torch.ones(1, device=DEV)
    for bad in ([t.half()], [t[::2]], [t, t.cpu()], [1.0]):
        with pytest.raises((TypeError, ValueError)):
            mb.mb_grad_norm(bad)
    with pytest.raises(ValueError):
        mb.mb_grad_clip([t], n, 1.0, out=[t, t])
    with pytest.raises(ValueError):
        mb.mb_grad_clip([t], torch.ones(2, device=DEV), 1.0)
    for ts, kw in (([t], dict(max_norm=0.0)), ([t], dict(max_norm=float("nan"))), ([t], dict(max_norm=1.0, out=[t[:99]])),
                   ([t[:99]], dict(max_norm=1.0, out=[t[1:]]))):
        with pytest.raises(mb.MbError):
            mb.mb_grad_clip(ts, n, **kw)
    with pytest.raises(mb.MbError):
        mb.mb_grad_norm([t], ws=torch.zeros(256, dtype=torch.uint8, device=DEV))
    with pytest.raises(mb.MbError):   # the norm among the gradients
        mb.mb_grad_norm([t], t[:1])
