"""mb_embed and mb_embed_backward against the 64-bit forms (oracle/train.py).

Bounds, u = 2^-24: a looked-up element is one fp32 product, rounded to the
output type (2^-9 for bf16). A gradient is a sum of fp32 terms in some order,
within (terms + 2) u of the sum of their magnitudes (the scaling and the
addition to an accumulated row are the other two). Twice over for slack."""
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

# tokens' shape, vocab, width, token type
CASES = [((1,), 1, 8, "u8"), ((3,), 256, 16, "i64"), ((2, 31), 5, 24, "i32"), ((64,), 256, 1024, "u8"), ((65,), 2, 520, "u8"),
         ((7, 129), 256, 64, "u8"), ((1003,), 300, 72, "i32"), ((4096,), 70000, 8, "i64"), ((4097,), 256, 264, "i64"),
         ((2, 8192), 256, 64, "u8"), ((40000,), 17, 8, "u8"), ((33000,), 32001, 16, "i32"), ((70001,), 256, 8, "u8"),
         ((100000,), 1000003, 8, "i64")]


def _tokens(shape, vocab, kind, seed=0, padding=0.1):
    g = np.random.default_rng(seed)
    n = int(np.prod(shape))
    t = np.minimum((vocab * g.random(n) ** 4).astype(np.int64), vocab - 1)   # low ids are frequent
    if kind != "u8":
        off = g.random(n) < padding
        t[off] = g.choice([-1, vocab, -100, vocab + 7, 2 ** 31 - 1], size=int(off.sum()))
    elif vocab < 256:
        t[g.random(n) < padding] = vocab
    return torch.from_numpy(t.reshape(shape)).to(TYPES[kind]).to(DEV)


def _rnd(*shape, dtype="f32", seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randn(*shape, device=DEV, generator=g).to(TYPES[dtype])


@pytest.mark.parametrize("case", CASES, ids=str)
@pytest.mark.parametrize("table, out", [("bf16", "f32"), ("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16")])
def test_lookup(case, table, out):
    shape, vocab, width, kind = case
    tok = _tokens(shape, vocab, kind)
    t = _rnd(vocab, width, dtype=table)
    for scale in (1.0, 11.3):
        o = torch.full((*shape, width), float("nan"), device=DEV, dtype=TYPES[out])
        mb.mb_embed(tok, t, o, scale=scale)
        ref = train.embed(tok.cpu().numpy(), to_np(t), float(np.float32(scale)))
        err = np.abs(to_np(o) - ref)
        assert np.all(err <= 2 * (U + (2.0 ** -9 if out == "bf16" else 0)) * np.abs(ref))
        if scale == 1.0 and table == "bf16":
            assert np.array_equal(to_np(o), ref)   # widened or copied, never rounded


@pytest.mark.parametrize("case", CASES, ids=str)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradient(case, dtype):
    shape, vocab, width, kind = case
    tok = _tokens(shape, vocab, kind, seed=1)
    dout = _rnd(*shape, width, dtype=dtype, seed=2)
    n, scale = tok.numel(), 1.7
    d = torch.full((vocab, width), float("nan"), device=DEV)
    mb.mb_embed_backward(tok, dout, d, scale=scale)
    s32, tn, dn = float(np.float32(scale)), tok.cpu().numpy(), to_np(dout)
    ref = train.embed_backward(tn, dn, vocab, s32)
    mag = train.embed_backward(tn, np.abs(dn), vocab, s32)
    terms = train.embed_backward(tn, np.ones((*shape, 1)), vocab)
    bound = 2 * (terms + 2) * U * mag
    assert np.all(np.abs(to_np(d) - ref) <= bound)
    # again, in a workspace that is not clear: the same to the last bit; then added to what is there
    ws = torch.full((mb.mb_embed_backward_workspace_size(n, vocab, width),), 255, dtype=torch.uint8, device=DEV)
    ws[:256] = 0
    two = torch.empty_like(d)
    mb.mb_embed_backward(tok, dout, two, scale=scale, ws=ws)
    assert torch.equal(d, two) and not ws[:256].any()
    start = _rnd(vocab, width, seed=3)
    acc = start.clone()
    mb.mb_embed_backward(tok, dout, acc, scale=scale, accumulate=True, ws=ws)
    s64 = to_np(start)
    assert np.all(np.abs(to_np(acc) - (s64 + ref)) <= bound + 2 * U * (np.abs(s64) + np.abs(ref)))
    absent = (terms[:, 0] == 0).nonzero()[0]
    assert np.array_equal(to_np(acc)[absent], s64[absent])


@pytest.mark.parametrize("n", [1, 63, 64, 65, 127, 128, 129, 191, 192, 193, 4095, 8193, 66000])
@pytest.mark.parametrize("pattern", ["one", "two", "last", "alternating", "none"])
def test_runs_and_pieces(n, pattern):
    # whole numbers: every order of the sum gives the same, exactly
    tok = torch.zeros(n, dtype=torch.int64, device=DEV)
    if pattern == "two":
        tok[n // 2:] = 9
    elif pattern == "last":
        tok[:] = 255
    elif pattern == "alternating":
        tok[1::2] = 3
    elif pattern == "none":
        tok[:] = -1
    dout = torch.arange(n, device=DEV)[:, None].remainder(17).float() - torch.arange(16, device=DEV)[None].float()
    d = torch.full((256, 16), 5.0, device=DEV)
    mb.mb_embed_backward(tok, dout, d)
    ref = torch.zeros_like(d)
    if pattern != "none":
        ref.index_add_(0, tok, dout)
    assert torch.equal(d, ref)


def test_gradient_is_the_difference_of_the_lookup():
    # the lookup is linear in the table: J(table + v) - J(table) is the gradient along v, up to fp32 rounding
    tok, table = _tokens((300,), 40, "i32", seed=4), _rnd(40, 32, seed=5)
    dout, v = _rnd(300, 32, seed=6), _rnd(40, 32, seed=7)

    def J(t):
        o = torch.empty(300, 32, device=DEV)
        mb.mb_embed(tok, t, o, scale=0.5)
        return float((o.double() * dout).sum())
    d = torch.empty_like(table)
    mb.mb_embed_backward(tok, dout, d, scale=0.5)
    along = float((d.double() * v).sum())
    assert abs(J(table + v) - J(table) - along) <= 1e-5 * float(d.norm() * v.norm())


def test_empty():
    d = torch.ones(4, 8, device=DEV)
    none = torch.empty(0, dtype=torch.int64, device=DEV)
    mb.mb_embed(none, d, torch.empty(0, 8, device=DEV))
    mb.mb_embed_backward(none, torch.empty(0, 8, device=DEV), d, accumulate=True)
    assert (d == 1).all()
    mb.mb_embed_backward(none, torch.empty(0, 8, device=DEV), d)
    assert not d.any()
    out = torch.ones(2, 8, device=DEV)
    mb.mb_embed(torch.zeros(2, dtype=torch.uint8, device=DEV), torch.empty(0, 8, device=DEV), out)
    assert not out.any()   # no table: every token is outside it


def test_nan_stays_in_its_row_and_column():
    tok = _tokens((5000,), 256, "u8", seed=8)
    dout = _rnd(5000, 24, seed=9)
    clean, hit = torch.empty(256, 24, device=DEV), torch.empty(256, 24, device=DEV)
    mb.mb_embed_backward(tok, dout, clean)
    dout[77, 3], dout[4000, 9] = float("nan"), float("inf")
    mb.mb_embed_backward(tok, dout, hit)
    same = torch.ones(256, 24, dtype=torch.bool, device=DEV)
    same[int(tok[77]), 3] = same[int(tok[4000]), 9] = False
    assert torch.equal(clean[same], hit[same]) and not torch.isfinite(hit[~same]).any()
    # rows of padding are not looked at
    pad = tok.to(torch.int32)
    pad[77] = pad[4000] = -1
    mb.mb_embed_backward(pad, dout, hit)
    assert torch.isfinite(hit).all()


def test_offsets_past_31_bits():
    n, W = 1 << 18, 8192   # 2^31 elements
    tok = torch.zeros(n, dtype=torch.uint8, device=DEV)
    tok[-1], tok[-2] = 200, 201
    table = _rnd(256, W, dtype="bf16", seed=10)
    out = torch.empty(n, W, device=DEV, dtype=torch.bfloat16)
    mb.mb_embed(tok, table, out)
    assert torch.equal(out[-1], table[200]) and torch.equal(out[-2], table[201]) and torch.equal(out[-3], table[0])
    d = torch.empty(256, W, device=DEV)
    out[:-2].zero_()
    mb.mb_embed_backward(tok, out, d)
    assert torch.equal(d[200], table[200].float()) and torch.equal(d[201], table[201].float()) and not d[:200].any()


def test_streams_graphs_and_the_plain_path():
    tok, dout, table = _tokens((3000,), 256, "u8"), _rnd(3000, 64), _rnd(256, 64, dtype="bf16")
    o, d = torch.empty(3000, 64, device=DEV), torch.empty(256, 64, device=DEV)
    mb.mb_embed(tok, table, o, scale=2.0)
    mb.mb_embed_backward(tok, dout, d, scale=2.0)
    torch.cuda.synchronize()
    s = torch.cuda.Stream(DEV)
    o2, d2 = torch.empty_like(o), torch.empty_like(d)
    ws = torch.zeros(mb.mb_embed_backward_workspace_size(3000, 256, 64), dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    mb.mb_embed(tok, table, o2, scale=2.0, stream=s)
    mb.mb_embed_backward(tok, dout, d2, scale=2.0, ws=ws, stream=s)
    s.synchronize()
    assert torch.equal(o, o2) and torch.equal(d, d2)
    d2.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mb.mb_embed_backward(tok, dout, d2, scale=2.0, ws=ws)
    graph.replay()
    graph.replay()
    assert torch.equal(d, d2)


def test_refusals():
    tok, table = torch.zeros(4, dtype=torch.uint8, device=DEV), torch.zeros(8, 16, device=DEV)
    out = torch.zeros(4, 16, device=DEV)
    for a in ((tok.float(), table, out), (tok, table.double(), out), (tok, table, out[:3]), (tok, table[:, ::2], out[:, :8]),
              (tok, table, out.half()), (tok.cpu(), table, out)):
        with pytest.raises((TypeError, ValueError)):
            mb.mb_embed(*a)
    with pytest.raises(mb.MbError):   # out over the table
        mb.mb_embed(tok, table, table[:4])
    with pytest.raises(mb.MbError):   # width % 8
        mb.mb_embed(tok, torch.zeros(8, 12, device=DEV), torch.zeros(4, 12, device=DEV))
    for a in ((tok, out, table.bfloat16()), (tok, out[:, :8], table), (tok, out.double(), table)):
        with pytest.raises((TypeError, ValueError)):
            mb.mb_embed_backward(*a)
    with pytest.raises(mb.MbError):   # workspace too small
        mb.mb_embed_backward(tok, out, table, ws=torch.zeros(256, dtype=torch.uint8, device=DEV))
