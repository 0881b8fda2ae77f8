"""Sizes at which parts of the training operators work that small cases do not
reach: the carried error of a long norm, masked rows that several CTAs share,
column tiles of the table's gradient.

Bounds, u = 2^-24. The norm of n equal elements: u of a square, 3 u of a group's
sum, 2 u of the carried sum, 5 u within a warp, halved by the root, and u of its
rounding: 6.5 u, taken as 8 (sums of these values without the carried error are
off by 30 u: 431 additions to a thread, most rounded the same way). Losses and
the table's gradient: those of test_cross_entropy_gpu.py and test_embed_gpu.py."""
import numpy as np
import pytest
import torch

import test_cross_entropy_gpu as ce
import test_embed_gpu as em
from oracle import train
from paper_2401_13660_gb300 import mbscan as mb

from _parity import to_np

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24


@pytest.mark.parametrize("value", [0.7, 1.7])
def test_norm_of_many_equal_elements(value):
    n = 1 << 28
    t = torch.full((n,), value, device=DEV)
    want = float(np.float32(value)) * 2.0 ** 14
    assert abs(float(mb.mb_grad_norm([t])) - want) <= 8 * U * want


@pytest.mark.parametrize("V", [1027, 8191, 20001, 40000, 131072])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masked_logits_of_long_rows(V, dtype):
    ce.test_masked_logits(V, dtype)   # eight rows: 1 to 8 CTAs to a row


@pytest.mark.parametrize("V", [8191, 20001, 40000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masked_logits_of_many_long_rows(V, dtype):
    # as many rows as leave one CTA to a row: each copy of a row as the oracle has it, and to the last bit as those that
    # begin at the same place of a 16-byte group (which the order of a row's sum goes by)
    logits, _, _ = ce._inputs(6, V, dtype, "i32", seed=11)
    low = torch.finfo(logits.dtype).min
    logits[0, 1::2] = -float("inf")
    logits[1, :-3] = -float("inf")
    logits[2, 4:] = low
    logits[3, :] = low
    logits[4, :] = -float("inf")
    logits[5, V // 2] = float("nan")
    tgt = torch.tensor([2, V - 1, 1, V // 2, 0, 3], device=DEV, dtype=torch.int32)
    n, places = 64, 16 // logits.element_size()
    many = logits.repeat(n, 1)
    loss, d = torch.full((6 * n,), 7.0, device=DEV), torch.full_like(many, 7.0)
    mb.mb_cross_entropy(many, tgt.repeat(n), loss, d)
    for x in (loss.view(torch.int32), d.view(torch.int16 if dtype == "bf16" else torch.int32)):
        x = x.reshape(n // places, places, -1)
        assert (x == x[0]).all()
    l, t = to_np(logits[:4]), tgt[:4].cpu().numpy()
    rl, rd = train.cross_entropy(l, t)
    bl, bd = ce._bounds(l, t, np.ones(4), 1.0, rl, rd, dtype)
    for i in range(0, 6 * places, 6):
        assert np.all(np.abs(to_np(loss[i:i + 4]) - rl) <= bl) and np.all(np.abs(to_np(d[i:i + 4]) - rd) <= bd)
        assert torch.isnan(loss[i + 4:i + 6]).all() and torch.isnan(d[i + 4:i + 6]).all()


@pytest.mark.parametrize("n, vocab, width, dtype", [(300, 5, 1040, "f32"), (3000, 256, 1792, "f32"), (9001, 3, 1792, "f32"),
                                                    (2000, 256, 2304, "f32"), (5000, 2, 2304, "bf16"), (700, 5000, 2056, "bf16"),
                                                    (1, 4, 4104, "f32"), (4000, 17, 4104, "bf16")])
@pytest.mark.parametrize("accumulate", [False, True])
def test_table_gradient_over_column_tiles(n, vocab, width, dtype, accumulate):
    # whole numbers: every order of the sum gives the same, exactly
    tok = em._tokens((n,), vocab, "i32", seed=n)
    g = torch.Generator(device=DEV).manual_seed(width)
    dout = torch.randint(-8, 9, (n, width), device=DEV, generator=g).to(em.TYPES[dtype])
    d = torch.randint(-8, 9, (vocab, width), device=DEV, generator=g).float()
    want = d.double() if accumulate else torch.zeros(vocab, width, device=DEV, dtype=torch.float64)
    ok = (tok >= 0) & (tok < vocab)
    want.index_add_(0, tok[ok].long(), dout[ok].double() * 2)
    mb.mb_embed_backward(tok, dout, d, scale=2.0, accumulate=accumulate)
    assert torch.equal(d.double(), want)


def test_table_gradient_of_a_large_vocabulary():
    # a subword table, tokens with the frequencies of text
    n, vocab, width = 8200, 32001, 1792
    g = np.random.default_rng(12)
    cum = np.cumsum(1.0 / np.arange(1, vocab + 1))
    t = g.permutation(vocab)[np.searchsorted(cum, g.random(n) * cum[-1]).clip(0, vocab - 1)]
    t[g.random(n) < 0.03] = -1
    tok, dout = torch.from_numpy(t).to(DEV), em._rnd(n, width, dtype="bf16", seed=13)
    d = torch.full((vocab, width), float("nan"), device=DEV)
    mb.mb_embed_backward(tok, dout, d)
    dn = to_np(dout)
    ref, mag = train.embed_backward(t, dn, vocab), train.embed_backward(t, np.abs(dn), vocab)
    terms = train.embed_backward(t, np.ones((n, 1)), vocab)
    assert np.all(np.abs(to_np(d) - ref) <= 2 * (terms + 2) * U * mag)
