"""Calls of the training operators back to back on one set of buffers, with
launch overlap: the results of chains without a synchronisation in between,
eagerly, from a CUDA graph and on two streams at once, equal those of the same
calls with one after each. And token counts beyond one tile of the sort."""
import numpy as np
import pytest
import torch

from oracle import train
from paper_2401_13660_gb300 import mbscan as mb

from _parity import to_np

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
B, L, D, V = 2, 300, 72, 256


class _Buffers:
    """Inputs, outputs and workspace of one chain: embed, convolution, its gradients, the table's, losses, clipping."""

    def __init__(self, seed):
        g = torch.Generator(device=DEV).manual_seed(seed)
        rnd = lambda *s, dtype=torch.float32: torch.randn(*s, device=DEV, generator=g).to(dtype)
        e = lambda *s, dtype=torch.float32: torch.empty(*s, device=DEV, dtype=dtype)
        self.tokens = torch.randint(0, V, (B, L), device=DEV, generator=g)
        self.table, self.w, self.bias = rnd(V, D), rnd(D, 4), rnd(D)
        self.x, self.out, self.state = e(B, L, D), e(B, L, D), rnd(B, 3, D)
        self.grads = dict(dx=e(B, L, D), dw=e(D, 4), dbias=e(D), dstate=e(B, 3, D))
        self.dtable, self.logits = rnd(V, D), rnd(B, L, V)
        self.loss = e(B, L)
        self.list = mb.mb_tensor_list([self.dtable, self.grads["dw"], self.grads["dbias"], self.logits])
        self.norm = e(1)
        n = max(mb.mb_conv1d_backward_workspace_size(B, L, D), mb.mb_embed_backward_workspace_size(B * L, V, D),
                mb.mb_grad_norm_workspace_size())
        self.ws = torch.zeros(n, dtype=torch.uint8, device=DEV)

    def calls(self):
        g = self.grads
        return [lambda: mb.mb_embed(self.tokens, self.table, self.x, scale=2.0),
                lambda: mb.mb_conv1d(self.x, self.w, self.out, bias=self.bias, state=self.state, state_out=self.state),
                lambda: mb.mb_conv1d_backward(self.x, self.w, self.out, bias=self.bias, state=self.state, dstate_out=self.state,
                                              grads=g, ws=self.ws),
                lambda: mb.mb_embed_backward(self.tokens, g["dx"], self.dtable, accumulate=True, ws=self.ws),
                lambda: mb.mb_cross_entropy(self.logits, self.tokens, self.loss, self.logits, scale=3.0),
                lambda: mb.mb_grad_norm(self.list, self.norm, ws=self.ws),
                lambda: mb.mb_grad_clip(self.list, self.norm, 4.0),
                lambda: mb.mb_embed(self.tokens, self.dtable, self.x, scale=0.5)]

    def all(self):
        return [self.x, self.out, self.state, *self.grads.values(), self.dtable, self.logits, self.loss, self.norm]


def _reference(seed, rounds):
    b = _Buffers(seed)
    for _ in range(rounds):
        for f in b.calls():
            f()
            torch.cuda.synchronize()
    return b


def _same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a.all(), b.all()))


def test_chained_calls():
    want = _reference(0, 12)
    b = _Buffers(0)
    for _ in range(12):
        for f in b.calls():
            f()
    torch.cuda.synchronize()
    assert _same(b, want) and not b.ws[:256].any()


def test_chain_in_a_graph():
    want = _reference(1, 7)
    b = _Buffers(1)
    for f in b.calls():   # one round eagerly, six replayed
        f()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        for f in b.calls():
            f()
    for _ in range(6):
        graph.replay()
    torch.cuda.synchronize()
    assert _same(b, want)


def test_chains_on_two_streams():
    want = [_reference(s, 8) for s in (2, 3)]
    bs, streams = [_Buffers(2), _Buffers(3)], [torch.cuda.Stream(DEV) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(8):
        for b, s in zip(bs, streams):
            with torch.cuda.stream(s):
                for f in b.calls():
                    f()
    torch.cuda.synchronize()
    assert _same(bs[0], want[0]) and _same(bs[1], want[1])


@pytest.mark.parametrize("n, vocab", [(131072, 256), (131073, 256), (300000, 70000), (400001, 3)])
def test_more_tokens_than_a_tile_of_each_sorting_cta(n, vocab):
    g = np.random.default_rng(n)
    tok = np.minimum((vocab * g.random(n) ** 3).astype(np.int64), vocab - 1)
    tok[g.random(n) < 0.05] = -1
    dout = g.integers(-8, 9, size=(n, 8)).astype(np.float32)   # whole numbers: exact in any order
    d = torch.empty(vocab, 8, device=DEV)
    mb.mb_embed_backward(torch.from_numpy(tok).to(DEV), torch.from_numpy(dout).to(DEV), d)
    assert np.array_equal(to_np(d), train.embed_backward(tok, dout, vocab))
