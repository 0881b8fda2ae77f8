"""mb_conv1d and mb_conv1d_backward against the 64-bit form (oracle/train.py).

Bounds, u = 2^-24. p is a sum of five fp32 terms: |dp| <= 5 u S with S the sum
of their magnitudes. SiLU's slope is at most 1.1, its own evaluation (exponential,
1 + e, quotient) is within 2^-20 (1 + |p|) relative. h = s (1 + p (1 - s)) has
slope at most 0.5 and is evaluated within (1 + |p|) 2^-21. A sum of n products is
within n u of the sum of their magnitudes, in any order. Each store to bf16 adds
half an ulp (2^-9). Every bound is taken twice over for slack; 1e-37 covers
results that the fp32 range flushes."""
import numpy as np
import pytest
import torch

from oracle import train
from paper_2401_13660_gb300 import mbscan as mb

from _parity import to_np

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
STORE = {"f32": 2.0 ** -24, "bf16": 2.0 ** -9}

# batch, L, width, dtype, wide, state, bias
CASES = [(1, 1, 8, "bf16", False, True, True), (2, 2, 16, "f32", True, True, False), (3, 3, 24, "bf16", True, False, True),
         (5, 4, 64, "f32", False, True, True), (1, 5, 264, "bf16", True, True, True), (2, 7, 40, "f32", False, False, False),
         (33, 16, 128, "bf16", False, True, True), (2, 63, 72, "bf16", True, True, True), (1, 64, 72, "f32", True, False, True),
         (3, 65, 8, "bf16", False, True, False), (2, 129, 520, "bf16", True, True, True), (1, 1003, 1544, "bf16", False, True, True),
         (2, 515, 264, "f32", True, True, True), (300, 1, 2048, "bf16", True, True, True), (2, 4099, 64, "bf16", False, False, True)]


def _inputs(b, L, D, dtype, wide, state, bias, seed=0, spread=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed + 7 * L + D)
    td = TYPES[dtype]
    rnd = lambda *s: spread * torch.randn(*s, device=DEV, generator=g)
    x = rnd(b, L, (2 if wide else 1) * D).to(td)[..., :D]
    return dict(x=x, w=torch.rand(D, 4, device=DEV, generator=g) - 0.5, bias=rnd(D) if bias else None,
                state=rnd(b, 3, D).to(td) if state else None, dout=rnd(b, L, D).to(td),
                dstate_out=rnd(b, 3, D).to(td) if state else None)


def _np(i):
    return {k: to_np(v) for k, v in i.items()}


def _check(got, ref, bound, what):
    err = np.abs(to_np(got) - ref)
    assert np.all(err <= bound), (what, float(np.max(err / bound)))


def _forward_bound(n, dtype):
    p, mag = train.conv1d_pre(n["x"], n["w"], n["bias"], n["state"])
    out, _ = train.conv1d(n["x"], n["w"], n["bias"], n["state"])
    return 2 * (1.1 * 5 * U * mag + (2.0 ** -20 * (1 + np.abs(p)) + STORE[dtype]) * np.abs(out)) + 1e-37


def _backward_bounds(n, r, dtype):
    p, mag = train.conv1d_pre(n["x"], n["w"], n["bias"], n["state"])
    w, L = np.abs(n["w"]), p.shape[1]
    eg = np.abs(n["dout"]) * (0.5 * 5 * U * mag + (1 + np.abs(p)) * 2.0 ** -21)
    g = np.abs(r["g"])
    u = np.abs(train._taps(n["x"], n["state"]))
    rows = p.shape[0] * L
    du, edw = np.zeros_like(u), np.zeros_like(w)
    for k in range(4):
        du[:, k:k + L] += w[:, k] * (eg + 6 * U * g)
        edw[:, k] = np.sum(eg * u[:, k:k + L] + (rows + 1) * U * g * u[:, k:k + L], axis=(0, 1))
    full = np.abs(np.concatenate([r["dstate"], r["dx"]], axis=1))
    du = 2 * (du + (STORE[dtype] + U) * full) + 1e-37
    return dict(dx=du[:, 3:], dstate=du[:, :3], dw=2 * edw + 1e-37,
                dbias=2 * np.sum(eg + rows * U * g, axis=(0, 1)) + 1e-37)


def _grads(i, **kw):
    return mb.mb_conv1d_backward(i["x"], i["w"], i["dout"], bias=i["bias"], state=i["state"],
                                 dstate_out=i["dstate_out"], **kw)


@pytest.mark.parametrize("case", CASES, ids=str)
def test_forward(case):
    i = _inputs(*case)
    n = _np(i)
    b, L, D = n["x"].shape
    out = torch.full((b, L, D), float("nan"), device=DEV, dtype=i["x"].dtype)
    so = torch.full((b, 3, D), float("nan"), device=DEV, dtype=i["x"].dtype)
    mb.mb_conv1d(i["x"], i["w"], out, bias=i["bias"], state=i["state"], state_out=so)
    ref, window = train.conv1d(n["x"], n["w"], n["bias"], n["state"])
    _check(out, ref, _forward_bound(n, case[3]), "out")
    assert np.array_equal(to_np(so), window)
    again = torch.empty_like(out)
    if i["state"] is not None:   # the window moved in place
        mb.mb_conv1d(i["x"], i["w"], again, bias=i["bias"], state=i["state"], state_out=i["state"])
        assert torch.equal(i["state"], so)
    else:
        mb.mb_conv1d(i["x"], i["w"], again, bias=i["bias"])
    assert torch.equal(out, again)


@pytest.mark.parametrize("case", CASES, ids=str)
def test_backward(case):
    i = _inputs(*case)
    n = _np(i)
    r = train.conv1d_backward(n["x"], n["w"], n["dout"], n["bias"], n["state"], n["dstate_out"])
    got = _grads(i)
    bounds = _backward_bounds(n, r, case[3])
    assert (got["dbias"] is None) == (i["bias"] is None) and (got["dstate"] is None) == (i["state"] is None)
    for k, v in got.items():
        if v is not None:
            _check(v, r[k], bounds[k], k)
    # given buffers (dx columns of wider rows), a reused workspace that is not clear: the same to the last bit
    b, L, D = n["x"].shape
    rows = torch.zeros(b, L, 3 * D, device=DEV, dtype=i["x"].dtype)
    g = dict(dx=rows[..., D:2 * D], dw=torch.empty(D, 4, device=DEV), dbias=torch.empty(D, device=DEV),
             dstate=torch.empty(b, 3, D, device=DEV, dtype=i["x"].dtype))
    ws = torch.full((mb.mb_conv1d_backward_workspace_size(b, L, D) + 64,), 255, dtype=torch.uint8, device=DEV)
    ws[:256] = 0
    two = _grads(i, grads=g, ws=ws)
    for k, v in got.items():
        assert v is None or torch.equal(two[k], v), k
    _check(two["dstate"], r["dstate"], bounds["dstate"], "dstate")
    _check(two["dbias"], r["dbias"], bounds["dbias"], "dbias")
    assert not rows[..., :D].any() and not rows[..., 2 * D:].any() and not ws[:256].any()


def test_gradient_is_the_difference_of_the_forward():
    # J = sum of out * dout with fp32 kernels: (J(a + e v) - J(a - e v)) / 2e against the gradient along v.
    # e = 2^-7: truncation e^2 |J'''| / 6, rounding of out 2^-23 |out dout| / e; both below 1e-3 of the norms' product.
    i = _inputs(2, 37, 64, "f32", False, True, True, seed=5)
    g = _grads(i)
    eps = 2.0 ** -7
    gen = torch.Generator(device=DEV).manual_seed(1)
    for name, key in (("x", "dx"), ("w", "dw"), ("bias", "dbias"), ("state", "dstate")):
        v = torch.randn(i[name].shape, device=DEV, generator=gen)

        def J(sign):
            j = dict(i, **{name: i[name] + sign * eps * v})
            out, so = torch.empty_like(j["x"]), torch.empty_like(j["state"])
            mb.mb_conv1d(j["x"], j["w"], out, bias=j["bias"], state=j["state"], state_out=so)
            return float((out.double() * i["dout"]).sum() + (so.double() * i["dstate_out"]).sum())
        along = float((g[key].double() * v).sum())
        assert abs((J(1) - J(-1)) / (2 * eps) - along) <= 1e-3 * float(g[key].double().norm() * v.double().norm())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_empty_spans_and_batches(dtype):
    i = _inputs(2, 0, 16, dtype, False, True, True)
    so = torch.empty_like(i["state"])
    mb.mb_conv1d(i["x"], i["w"], i["x"].clone(), bias=i["bias"], state=i["state"], state_out=so)
    assert torch.equal(so, i["state"])
    mb.mb_conv1d(i["x"], i["w"], i["x"].clone(), bias=i["bias"], state_out=so)
    assert not so.any()
    g = _grads(i)
    assert torch.equal(g["dstate"], i["dstate_out"]) and not g["dw"].any() and not g["dbias"].any()
    e = _inputs(0, 5, 16, dtype, False, True, True)
    g = _grads(e, grads=dict(dw=torch.ones(16, 4, device=DEV), dbias=torch.ones(16, device=DEV)))
    assert not g["dw"].any() and not g["dbias"].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_prompt_then_steps_is_one_span(dtype):
    i = _inputs(3, 90, 128, dtype, False, True, True, seed=2)
    whole = torch.empty_like(i["x"])
    mb.mb_conv1d(i["x"], i["w"], whole, bias=i["bias"], state=i["state"])
    window, first = i["state"].clone(), i["x"][:, :77].contiguous()
    out = torch.empty_like(first)
    mb.mb_conv1d(first, i["w"], out, bias=i["bias"], state=window, state_out=window)
    assert torch.equal(out, whole[:, :77])
    n = _np(i)
    bound = _forward_bound(n, dtype)
    ref, _ = train.conv1d(n["x"], n["w"], n["bias"], n["state"])
    for t in range(77, 90):
        y = torch.empty(3, 128, device=DEV, dtype=i["x"].dtype)
        mb.mb_conv1d_step(i["x"][:, t].contiguous(), window, i["w"], y, bias=i["bias"])
        _check(y, ref[:, t], 4 * bound[:, t], "step")   # the step evaluates SiLU on the SFU for both types


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_infinities_and_nan_stay_in_their_channel_and_steps(dtype):
    i = _inputs(1, 200, 32, dtype, False, True, True, seed=3)
    clean = torch.empty_like(i["x"])
    mb.mb_conv1d(i["x"], i["w"], clean, bias=i["bias"], state=i["state"])
    gc = _grads(i)
    x = i["x"].clone()
    x[0, 100, 5], x[0, 150, 9] = float("nan"), float("inf")
    out = torch.empty_like(x)
    mb.mb_conv1d(x, i["w"], out, bias=i["bias"], state=i["state"])
    hit = torch.zeros_like(x, dtype=torch.bool)
    hit[0, 100:104, 5] = hit[0, 150:154, 9] = True
    assert torch.equal(out[~hit], clean[~hit]) and torch.isnan(out[0, 100:104, 5]).all()
    gn = _grads(dict(i, x=x))
    near = torch.zeros_like(hit)
    near[0, 97:104, 5] = near[0, 147:154, 9] = True
    assert torch.equal(gn["dx"][~near], gc["dx"][~near])
    others = [c for c in range(32) if c not in (5, 9)]
    assert torch.equal(gn["dw"][others], gc["dw"][others])


def test_large_arguments():
    # p of +-300: out = p or a flushed zero, slope 1 or 0, nothing overflows
    i = _inputs(1, 40, 16, "f32", False, True, True, seed=4, spread=300.0)
    n = _np(i)
    out = torch.empty_like(i["x"])
    mb.mb_conv1d(i["x"], i["w"], out, bias=i["bias"], state=i["state"])
    _check(out, train.conv1d(n["x"], n["w"], n["bias"], n["state"])[0], _forward_bound(n, "f32"), "out")
    r = train.conv1d_backward(n["x"], n["w"], n["dout"], n["bias"], n["state"], n["dstate_out"])
    bounds = _backward_bounds(n, r, "f32")
    for k, v in _grads(i).items():
        _check(v, r[k], bounds[k], k)


def test_offsets_past_32_bits():
    # 2^31 - 2^20 elements of columns in rows twice as wide: the last rows' offsets pass 2^32
    b, L, D = 1, (1 << 20) - 512, 2048
    x = torch.zeros(b, L, 2 * D, device=DEV, dtype=torch.bfloat16)
    i = _inputs(1, 300, D, "bf16", False, False, True, seed=6)
    x[:, -300:, :D] = i["x"]
    out = torch.empty(b, L, D, device=DEV, dtype=torch.bfloat16)
    mb.mb_conv1d(x[..., :D], i["w"], out, bias=i["bias"])
    ref = torch.empty_like(i["x"])
    mb.mb_conv1d(i["x"], i["w"], ref, bias=i["bias"])
    assert torch.equal(out[:, -300:], ref)
    dx = x   # the gradient's columns beside the inputs'
    dout = out.zero_()
    dout[:, -300:] = i["dout"]
    g = mb.mb_conv1d_backward(x[..., :D], i["w"], dout, bias=i["bias"],
                              grads=dict(dx=torch.empty_like(x)[..., D:]))
    small = mb.mb_conv1d_backward(i["x"], i["w"], i["dout"], bias=i["bias"])
    assert torch.equal(g["dx"][:, -300:], small["dx"])
    assert float((g["dw"] - small["dw"]).abs().max()) <= 1e-4 * float(small["dw"].abs().max())


def test_streams_and_native_marshalling():
    i = _inputs(2, 33, 64, "bf16", True, True, True)
    want, wg = torch.empty(2, 33, 64, device=DEV, dtype=torch.bfloat16), None
    mb.mb_conv1d(i["x"], i["w"], want, bias=i["bias"], state=i["state"])
    wg = _grads(i)
    torch.cuda.synchronize()
    s = torch.cuda.Stream(DEV)
    out = torch.empty_like(want)
    mb.mb_conv1d(i["x"], i["w"], out, bias=i["bias"], state=i["state"], stream=s)   # the plain path
    g = _grads(i, stream=s)
    s.synchronize()
    assert torch.equal(out, want) and all(torch.equal(g[k], wg[k]) for k in wg)
    graph = torch.cuda.CUDAGraph()
    out.zero_()
    with torch.cuda.graph(graph):
        mb.mb_conv1d(i["x"], i["w"], out, bias=i["bias"], state=i["state"])
    graph.replay()
    assert torch.equal(out, want)


def test_refusals():
    i = _inputs(2, 8, 16, "bf16", False, True, True)
    out = torch.empty_like(i["x"])
    bad = [dict(x=i["x"].half()), dict(w=i["w"][:, :3].contiguous()), dict(out=out[:, :7]), dict(state=i["state"].float()),
           dict(bias=i["bias"].double()), dict(state_out=i["state"][:1]), dict(x=i["x"].transpose(0, 1))]
    for kw in bad:
        a = dict(dict(x=i["x"], w=i["w"], out=out, bias=i["bias"], state=i["state"]), **kw)
        with pytest.raises((TypeError, ValueError)):
            mb.mb_conv1d(a.pop("x"), a.pop("w"), a.pop("out"), **a)
    with pytest.raises(mb.MbError):   # out over x
        mb.mb_conv1d(i["x"], i["w"], i["x"], bias=i["bias"])
    with pytest.raises(mb.MbError):   # width % 8
        y = torch.zeros(1, 2, 12, device=DEV)
        mb.mb_conv1d(y, torch.zeros(12, 4, device=DEV), torch.empty_like(y))
    with pytest.raises(mb.MbError):   # workspace too small
        _grads(i, ws=torch.zeros(256, dtype=torch.uint8, device=DEV))
