"""The decoder on 8-bit projections: every 8-bit step of every block against the definition in 64 bits, from the block's
own traced inputs; graphs; drawing bytes."""
import numpy as np
import pytest
import torch

from oracle import serve
from paper_2401_13660_gb300.decoder import CONFIGS, Decoder, DecoderConfig

from _parity import to_np

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _product_bound(a, w, want):
    """Sums of a.shape[1] products in fp32, in any order, and bf16 once (see test_matmul_q8_gpu.py)."""
    return a.shape[1] * 2.0 ** -23 * (np.abs(a) @ np.abs(w).T) * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want)


def _values(x, block_rows):
    q, s = serve.quantize(x, block_rows)
    return q * serve.factors(s, block_rows, *x.shape)


@pytest.mark.parametrize("cfg, batch", [(CONFIGS["tiny_2x64"], 5), (DecoderConfig(n_layers=1, d_model=1024, d_inner=2048, dt_rank=64), 33)])
def test_every_block(cfg, batch):
    plain = Decoder(cfg, batch=batch, device=DEV, seed=3)
    dec = Decoder(cfg, batch=batch, device=DEV, seed=3, bits=8)
    assert dec.bytes_per_step() < plain.bytes_per_step()
    trace = []
    g = torch.Generator(device=DEV).manual_seed(9)
    for _ in range(2):
        dec.step(torch.randint(0, 256, (batch,), device=DEV, generator=g), trace=trace)
    dec.check()
    for i, t in enumerate(trace):
        L = plain.layers[i % cfg.n_layers]
        W_in, W_out = _values(to_np(L["W_in"]).reshape(2 * cfg.d_inner, -1), 128), _values(to_np(L["W_out"]), 128)
        kept = dec.layers[i % cfg.n_layers]
        assert np.array_equal(to_np(kept["W_in"].values()), W_in) and np.array_equal(to_np(kept["W_out"].values()), W_out)
        h = _values(serve.rmsnorm(to_np(t["residual_out"]), to_np(L["norm_w"]), float(np.float32(cfg.eps))), 1)
        assert np.array_equal(to_np(t["h"]), h)
        xz = np.concatenate([to_np(t["x"]), to_np(t["z"])], 1)
        assert (np.abs(xz - h @ W_in.T) <= _product_bound(h, W_in, h @ W_in.T)).all()
        y = _values(to_np(t["y"]), 1)
        assert np.array_equal(to_np(t["y8"]), y)
        assert (np.abs(to_np(t["out"]) - y @ W_out.T) <= _product_bound(y, W_out, y @ W_out.T)).all()


def test_graph_replay_equals_eager_and_draws():
    a, b = (Decoder(CONFIGS["tiny_2x64"], batch=8, device=DEV, seed=4, bits=8) for _ in range(2))
    b.capture()
    u = torch.rand(6, 8, device=DEV)
    start = torch.arange(8, device=DEV)
    x = a.generate(start, u, temperature=0.8, top_k=20, top_p=0.9, min_p=0.01)
    y = b.generate(start, u, temperature=0.8, top_k=20, top_p=0.9, min_p=0.01)
    assert torch.equal(x, y) and int(x.min()) >= 0 and int(x.max()) < 256
    for s, t in zip(a.ssm + a.conv, b.ssm + b.conv):
        assert torch.equal(s, t)
    l, last = to_np(a.logits), to_np(u[-1])
    for r in range(8):
        assert serve.sample(l[r], last[r], temperature=float(np.float32(0.8)), top_k=20, top_p=float(np.float32(0.9)),
                            min_p=float(np.float32(0.01)))[0] == int(x[-1, r])


def test_draw_settings_of_their_own():
    dec = Decoder(CONFIGS["tiny_2x64"], batch=4, device=DEV, seed=4)
    dec.step(torch.arange(4, device=DEV))
    u, prob = torch.rand(4, device=DEV), torch.empty(4, device=DEV)
    best = dec.draw(u, temperature=0.0, prob=prob).clone()
    assert torch.equal(best, dec.logits.float().argmax(1)) and (prob == 1).all()
    assert torch.equal(dec.draw(u, top_k=torch.ones(4, dtype=torch.int32, device=DEV)), best)


def test_refusals():
    with pytest.raises(ValueError, match="bits"):
        Decoder(CONFIGS["tiny_2x64"], batch=1, device=DEV, bits=4)
    with pytest.raises(ValueError, match="no 8-bit projections"):
        Decoder(DecoderConfig(n_layers=1, d_model=64, d_inner=64, dt_rank=8), batch=1, device=DEV, bits=8)
