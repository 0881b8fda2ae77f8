"""The 8-bit operators and the draw as they are used: one after the other on one stream without a wait between, captured
and replayed, on streams of their own, on two streams at once, and through the Python path of the binding."""
import numpy as np
import pytest
import torch

from oracle import serve
from paper_2401_13660_gb300 import mbscan as mb

from _parity import to_np

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
E4M3 = torch.float8_e4m3fn


class Chain:
    """norm -> product -> quantise -> product -> draw, all buffers its own."""

    def __init__(self, rows, width, inner, vocab, seed):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.residual0 = torch.randn(rows, width, device=DEV, generator=g)
        self.add = torch.randn(rows, width, device=DEV, generator=g).bfloat16()
        self.w = torch.rand(width, device=DEV, generator=g) + 0.5
        self.u = torch.rand(rows, device=DEV, generator=g)
        self.top_p = torch.full((rows,), 0.9, device=DEV)
        self.W1, self.W2 = (torch.randn(a, b, device=DEV, generator=g) / b ** 0.5 for a, b in ((inner, width), (vocab, inner)))
        st = serve.stride
        u8 = dict(dtype=torch.uint8, device=DEV)
        self.residual = torch.empty_like(self.residual0)
        self.h, self.hs = torch.empty(rows, width, dtype=E4M3, device=DEV), torch.empty(rows, st(width), **u8)
        self.y, self.ys = torch.empty(rows, inner, dtype=E4M3, device=DEV), torch.empty(rows, st(inner), **u8)
        self.q1, self.s1 = torch.empty(inner, width, dtype=E4M3, device=DEV), torch.empty(-(-inner // 128), st(width), **u8)
        self.q2, self.s2 = torch.empty(vocab, inner, dtype=E4M3, device=DEV), torch.empty(-(-vocab // 128), st(inner), **u8)
        self.mid = torch.empty(rows, inner, dtype=torch.bfloat16, device=DEV)
        self.logits = torch.empty(rows, vocab, device=DEV)
        self.tokens, self.prob = torch.empty(rows, dtype=torch.int64, device=DEV), torch.empty(rows, device=DEV)
        self.ws = torch.zeros(256, **u8)

    def outputs(self):
        return [self.residual, self.h.view(torch.uint8), self.hs, self.mid, self.y.view(torch.uint8), self.ys, self.logits,
                self.tokens, self.prob]

    def run(self, stream=None):
        k = dict(stream=stream)
        mb.mb_quantize_q8(self.W1, self.q1, self.s1, block_rows=128, **k)
        mb.mb_quantize_q8(self.W2, self.q2, self.s2, block_rows=128, **k)
        self.residual.copy_(self.residual0)
        mb.mb_rmsnorm_q8(self.residual, self.w, self.h, self.hs, add=self.add, **k)
        mb.mb_matmul_q8(self.h, self.hs, self.q1, self.s1, self.mid, ws=self.ws, **k)
        mb.mb_quantize_q8(self.mid, self.y, self.ys, **k)
        mb.mb_matmul_q8(self.y, self.ys, self.q2, self.s2, self.logits, ws=self.ws, **k)
        mb.mb_sample(self.logits, self.u, self.tokens, top_p=self.top_p, prob=self.prob, **k)

    def want(self):
        """Step by step from each step's own inputs, but for the products' sums."""
        r = to_np(self.residual0 + self.add.float())
        assert np.array_equal(to_np(self.residual), r)
        q, s = serve.quantize(serve.rmsnorm(r, to_np(self.w), float(np.float32(1e-5))), 1)
        assert np.array_equal(serve.e4m3_values(self.h.view(torch.uint8).cpu().numpy()), q) and np.array_equal(self.hs.cpu().numpy(), s)
        q, s = serve.quantize(to_np(self.mid), 1)
        assert np.array_equal(serve.e4m3_values(self.y.view(torch.uint8).cpu().numpy()), q) and np.array_equal(self.ys.cpu().numpy(), s)
        for a, sa, w, sw, out, half in ((self.h, self.hs, self.q1, self.s1, self.mid, 2.0 ** -8),
                                        (self.y, self.ys, self.q2, self.s2, self.logits, 2.0 ** -24)):
            ref, size = serve.matmul(*(t.view(torch.uint8).cpu().numpy() for t in (a, sa, w, sw)))
            assert (np.abs(to_np(out) - ref) <= a.shape[1] * 2.0 ** -23 * size * (1 + half) + half * np.abs(ref)).all()
        l, u, tokens = to_np(self.logits), to_np(self.u), self.tokens.cpu().numpy()
        for i in range(0, len(u), 1 + len(u) // 40):
            p = float(np.float32(0.9))
            near = {serve.sample(l[i], u[i] + d, top_p=p * (1 + e))[0] for d in (-2.0 ** -30, 0, 2.0 ** -30) for e in (-2.0 ** -30, 0, 2.0 ** -30)}
            assert tokens[i] in near


SIZES = [(1, 64, 128, 256), (33, 272, 400, 1000), (256, 1024, 2048, 256), (1500, 512, 1040, 264)]


@pytest.mark.parametrize("size", SIZES, ids=str)
def test_one_after_the_other(size):
    c = Chain(*size, seed=1)
    c.run()
    c.want()
    first = [t.clone() for t in c.outputs()]
    for _ in range(20):
        c.run()
    for t, f in zip(c.outputs(), first):
        assert torch.equal(t, f)
    assert mb.mb_check(c.ws)[0] == mb.MB_OK


@pytest.mark.parametrize("size", SIZES, ids=str)
def test_captured(size):
    c = Chain(*size, seed=2)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        c.run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.run()
    c.residual0.normal_()
    c.u.uniform_()
    for t in c.outputs():
        t.zero_()
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    c.want()


def test_streams_at_once():
    """Two chains on streams of their own, the stream given or current, while a third runs on the default one."""
    chains = [Chain(*size, seed=3 + i) for i, size in enumerate([SIZES[2], SIZES[1], SIZES[3]])]
    s = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        with torch.cuda.stream(s[0]):
            chains[0].run()
        with torch.cuda.stream(s[1]):
            chains[1].run(stream=s[1])
        chains[2].run()
    torch.cuda.synchronize()
    for c in chains:
        c.want()


def test_python_path_gives_the_same(monkeypatch):
    a, b = Chain(*SIZES[1], seed=9), Chain(*SIZES[1], seed=9)
    a.run()
    monkeypatch.setattr(mb, "_fast", mb._Declined())
    b.run()
    for x, y in zip(a.outputs(), b.outputs()):
        assert torch.equal(x, y)


def test_refused_calls_launch_nothing():
    c = Chain(*SIZES[1], seed=5)
    c.run()
    before = [t.clone() for t in c.outputs()]
    with pytest.raises(ValueError):
        mb.mb_matmul_q8(c.h, c.hs, c.q2, c.s2, c.logits)
    with pytest.raises(mb.MbError):   # scales on top of the values
        mb.mb_quantize_q8(c.mid, c.y, c.y.view(torch.uint8).view(-1)[:33 * 4].view(33, 4))
    for t, f in zip(c.outputs(), before):
        assert torch.equal(t, f)
