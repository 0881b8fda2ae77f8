"""Tokens outside the vocabulary in the whole-model decoder: looked up as zeros,
without an effect on the other streams."""
import pytest
import torch

from paper_2401_13660_gb300.decoder import CONFIGS, Decoder

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("bad", [-1, 256, 1 << 40, -(1 << 40)])
@pytest.mark.parametrize("captured", [False, True])
def test_a_token_outside_the_vocabulary_is_zeros(bad, captured):
    a, b = (Decoder(CONFIGS["tiny_2x64"], 8, DEV, seed=3) for _ in range(2))
    if captured:
        a.capture(), b.capture()
    b.emb[7] = 0   # what stream 5 of b looks up instead
    a.emb[7] = 0   # (the head has these rows too)
    g = torch.Generator(device=DEV).manual_seed(2)
    for _ in range(3):
        tokens = torch.randint(8, 256, (8,), device=DEV, generator=g)
        x, y = tokens.clone(), tokens.clone()
        x[5], y[5] = bad, 7
        assert torch.equal(a.step(x), b.step(y))
    assert torch.equal(a.residual[5], b.residual[5]) and torch.isfinite(a.logits).all()
    a.check()
    b.check()
