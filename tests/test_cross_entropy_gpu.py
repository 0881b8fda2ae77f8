"""mb_cross_entropy against the 64-bit form (oracle/train.py).

Bounds, u = 2^-24. A term exp(l - m) carries the rounding of its argument
((m - l) u, twice on the SFU path, where it is also scaled by log2 e) and of
the exponential (4 u). A sum goes through chains of at most V/256 + 64
additions, each of which may also rescale: 4 u a link. So s is within
rel = u (4 (V/256 + 64) + 16 + 2 sum p (m - l)) of its value, the loss within
rel + u (|m - l_y| + |log s| + |loss|), and p within rel + u (2 (m - l) + 8) of
p. dlogits adds u for its difference and half an ulp (2^-9) when it is bf16.
Twice over for slack; 1e-37 covers what the fp32 range flushes."""
import numpy as np
import pytest
import torch

from oracle import train
from paper_2401_13660_gb300 import mbscan as mb

from _parity import to_np

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "u8": torch.uint8, "i32": torch.int32, "i64": torch.int64}

CASES = [(1, 1, "f32", "u8"), (3, 2, "bf16", "u8"), (1, 256, "bf16", "u8"), (9, 256, "f32", "i64"), (1000, 256, "bf16", "u8"),
         (17, 255, "bf16", "i32"), (17, 257, "f32", "i32"), (5, 250, "f32", "u8"), (8, 264, "bf16", "i64"), (7, 1024, "bf16", "i64"),
         (7, 1023, "f32", "i32"), (7, 1025, "bf16", "i64"), (3, 2048, "f32", "i32"), (4, 8000, "bf16", "i64"),
         (5, 32001, "bf16", "i64"), (3, 50257, "f32", "i64"), (2, 200003, "bf16", "i32"), (2, 131072, "f32", "i64")]


def _inputs(n, V, dtype, kind, seed=0, spread=3.0):
    g = torch.Generator(device=DEV).manual_seed(seed + n + V)
    logits = (spread * torch.randn(n, V, device=DEV, generator=g)).to(TYPES[dtype])
    tgt = torch.randint(0, V, (n,), device=DEV, generator=g).clamp(max=255 if kind == "u8" else V)
    if kind != "u8" and n > 4:
        tgt[1], tgt[3] = -100, V
    weight = torch.rand(n, device=DEV, generator=g)
    if n > 2:
        weight[2] = 0.0
    return logits, tgt.to(TYPES[kind]), weight


def _bounds(l, tgt, w, scale, loss, d, dtype):
    n, V = l.shape
    finite = np.isfinite(l)
    m = np.max(l, axis=1, keepdims=True)
    gap = np.where(finite, m - np.where(finite, l, 0), 0.0)
    e = np.where(finite, np.exp(-gap), 0.0)
    s = e.sum(1, keepdims=True)
    p = e / s
    rel = U * (4 * (V / 256 + 64) + 16 + 2 * np.sum(p * gap, 1, keepdims=True))
    safe = np.where((tgt >= 0) & (tgt < V), tgt, 0)
    at = np.take_along_axis(gap, safe[:, None], 1)
    w = np.where((tgt >= 0) & (tgt < V), w, 0.0)[:, None]
    bl = 2 * w * (rel + U * (at + np.abs(np.log(s)))) + 2 * U * np.abs(loss[:, None])
    hot = np.zeros_like(p)
    np.put_along_axis(hot, safe[:, None], 1.0, 1)
    bd = 2 * np.abs(w * scale) * (p * (rel + U * (2 * gap + 8)) + 3 * U * np.abs(p - hot))
    return bl[:, 0] + 1e-37, bd + 2 * (2.0 ** -9 if dtype == "bf16" else U) * np.abs(d) + 1e-37


@pytest.mark.parametrize("case", CASES, ids=str)
@pytest.mark.parametrize("weighted", [False, True])
def test_loss_and_gradient(case, weighted):
    n, V, dtype, kind = case
    logits, tgt, weight = _inputs(*case)
    w = weight if weighted else None
    loss = torch.full((n,), float("nan"), device=DEV)
    d = torch.full_like(logits, float("nan"))
    mb.mb_cross_entropy(logits, tgt, loss, d, weight=w, scale=1.0 / n)
    l, t = to_np(logits), tgt.cpu().numpy().astype(np.int64)
    scale = float(np.float32(1.0 / n))
    w64 = np.ones(n) if w is None else to_np(w)
    rl, rd = train.cross_entropy(l, t, w64, scale)
    bl, bd = _bounds(l, t, w64, scale, rl, rd, dtype)
    assert np.all(np.abs(to_np(loss) - rl) <= bl), float(np.max(np.abs(to_np(loss) - rl) / bl))
    assert np.all(np.abs(to_np(d) - rd) <= bd), float(np.max(np.abs(to_np(d) - rd) / bd))
    # without the gradient, and over the logits: the same to the last bit
    again = torch.empty_like(loss)
    mb.mb_cross_entropy(logits, tgt, again, weight=w)
    assert torch.equal(loss, again)
    mb.mb_cross_entropy(logits, tgt, again, logits, weight=w, scale=1.0 / n)
    assert torch.equal(loss, again) and torch.equal(logits, d)


def test_gradient_is_the_difference_of_the_loss():
    # central differences of the fp32 losses, e = 2^-6 along one logit each: e^2/6 of the third derivative
    # (below 0.1) is 4e-6, rounding of a loss below 10 is 1e-6 / e = 6e-5
    logits, tgt, _ = _inputs(40, 256, "f32", "u8", seed=3, spread=1.0)
    loss, d = torch.empty(40, device=DEV), torch.empty_like(logits)
    mb.mb_cross_entropy(logits, tgt, loss, d)
    eps = 2.0 ** -6
    for v in (0, 100, 255, int(tgt[7])):
        side = []
        for sign in (1, -1):
            x, o = logits.clone(), torch.empty_like(loss)
            x[:, v] += sign * eps
            mb.mb_cross_entropy(x, tgt, o)
            side.append(o.double())
        assert float(((side[0] - side[1]) / (2 * eps) - d[:, v]).abs().max()) <= 2e-4


@pytest.mark.parametrize("V", [8, 256, 1000, 5000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masked_logits(V, dtype):
    logits, tgt, _ = _inputs(8, V, dtype, "i32", seed=4)
    tgt = torch.arange(8, device=DEV, dtype=torch.int32) % V
    low = torch.finfo(logits.dtype).min
    logits[0, ::2] = -float("inf")      # masked tokens; the target among them
    logits[1, 3:] = -float("inf")
    logits[2, 4:] = low                 # the type's lowest value
    logits[3, :] = low                  # all of it: uniform
    logits[4, :] = -float("inf")        # no distribution
    logits[5, 1] = float("nan")
    logits[6, :] = float("nan")         # not looked at: weight 0
    logits[7, :] = float("inf")         # not looked at: no target
    tgt[7] = -1
    weight = torch.ones(8, device=DEV)
    weight[6] = 0.0
    loss, d = torch.full((8,), 7.0, device=DEV), torch.full_like(logits, 7.0)
    mb.mb_cross_entropy(logits, tgt, loss, d, weight=weight)
    assert loss[0] == float("inf") and (d[0, 2::2] == 0).all() and torch.isfinite(d[0]).all() and d[0, 0] == -1
    l, t = to_np(logits[1:4]), tgt[1:4].cpu().numpy()
    rl, rd = train.cross_entropy(l, t)
    bl, bd = _bounds(l, t, np.ones(3), 1.0, rl, rd, dtype)
    assert np.all(np.abs(to_np(loss[1:4]) - rl) <= bl) and np.all(np.abs(to_np(d[1:4]) - rd) <= bd)
    for r in (4, 5):
        assert torch.isnan(loss[r]) and torch.isnan(d[r]).all()
    for r in (6, 7):
        assert loss[r] == 0 and (d[r] == 0).all()


def test_large_logits_and_certain_targets():
    x = torch.full((3, 256), -1e4, device=DEV)
    x[0, 5], x[1, 5], x[2, 5] = 3e38, 1e4, 1e4
    tgt = torch.tensor([5, 5, 6], device=DEV, dtype=torch.uint8)
    loss, d = torch.empty(3, device=DEV), torch.empty_like(x)
    mb.mb_cross_entropy(x, tgt, loss, d)
    assert loss.tolist() == [0.0, 0.0, 2e4] and not d[:2].any() and d[2, 5] == 1 and d[2, 6] == -1


def test_shapes_streams_graphs_and_empty():
    logits, tgt, _ = _inputs(60, 256, "bf16", "u8", seed=5)
    loss, d = torch.empty(60, device=DEV), torch.empty_like(logits)
    mb.mb_cross_entropy(logits, tgt, loss, d, scale=0.5)
    l2, d2 = torch.empty(4, 15, device=DEV), torch.empty(4, 15, 256, device=DEV, dtype=torch.bfloat16)
    torch.cuda.synchronize()
    s = torch.cuda.Stream(DEV)
    mb.mb_cross_entropy(logits.view(4, 15, 256), tgt.view(4, 15), l2, d2, scale=0.5, stream=s)
    s.synchronize()
    assert torch.equal(l2.view(-1), loss) and torch.equal(d2.view(60, 256), d)
    l2.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mb.mb_cross_entropy(logits.view(4, 15, 256), tgt.view(4, 15), l2, d2, scale=0.5)
    graph.replay()
    assert torch.equal(l2.view(-1), loss)
    mb.mb_cross_entropy(logits[:0], tgt[:0], loss[:0], d[:0])


def test_offsets_past_31_bits():
    n, V = 65535, 32768
    logits = torch.zeros(n, V, device=DEV, dtype=torch.bfloat16)
    logits[-1, 7] = 20.0
    tgt = torch.full((n,), 7, device=DEV, dtype=torch.int32)
    loss = torch.empty(n, device=DEV)
    mb.mb_cross_entropy(logits, tgt, loss, logits)
    want = float(np.log(1 + (V - 1) * np.exp(-20.0)))
    assert abs(float(loss[-1]) - want) <= 1e-6 and abs(float(loss[-2]) - np.log(V)) <= 1e-5
    assert float(logits[-2, 7]) == -1.0 and abs(float(logits[-2, 9]) * V - 1) <= 2.0 ** -8


def test_refusals():
    logits, tgt, w = _inputs(6, 256, "f32", "i64")
    loss, d = torch.empty(6, device=DEV), torch.empty_like(logits)
    for a, kw in (((logits.half(), tgt, loss), {}), ((logits, tgt.float(), loss), {}), ((logits, tgt[:5], loss), {}),
                  ((logits, tgt, loss.double()), {}), ((logits[:, ::2], tgt, loss), {}), ((logits, tgt, loss, d.bfloat16()), {}),
                  ((logits, tgt, loss, d), dict(weight=w[:5])), ((logits, tgt.cpu(), loss), {})):
        with pytest.raises((TypeError, ValueError)):
            mb.mb_cross_entropy(*a, **kw)
    with pytest.raises(mb.MbError):   # losses inside the logits
        mb.mb_cross_entropy(logits, tgt, logits.view(-1)[:6])


@pytest.mark.parametrize("V", [4096, 4097, 8191, 8192, 8193, 16384, 16385])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [3, 70, 310])
def test_sizes_where_rows_change_hands(n, V, dtype):
    # rows kept in the registers of 128 or 256 threads, read twice, by one CTA or several
    test_loss_and_gradient((n, V, dtype, "i64"), True)
