"""The training example's autograd functions (trainer.py): what they round, and
how often."""
import numpy as np
import pytest
import torch

from oracle import train
from paper_2401_13660_gb300 import trainer as tr

from _parity import to_np

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dloss", [1.0, 1 / 3, -2.7, 0.0])
def test_gradient_of_a_scaled_loss_is_rounded_once(dtype, dloss):
    # Logits within 16 of the largest: a probability is within rel = 2^-13 of its value (3e-5 by the kernel's bounds).
    # What is stored lies between the roundings of the ends of that interval.
    g = torch.Generator(device=DEV).manual_seed(4)
    logits = (16 * torch.rand(64, 256, device=DEV, generator=g)).to(dtype).requires_grad_()
    targets = torch.randint(0, 256, (64,), device=DEV, generator=g)
    targets[5] = -1
    scale = 1.0 / 64
    loss = tr.CrossEntropy.apply(logits, targets, scale)
    (loss * dloss).backward()
    c = float(np.float32(dloss))
    rl, rd = train.cross_entropy(to_np(logits), targets.cpu().numpy(), scale=scale * c)
    hot = np.zeros_like(rd)
    ok = to_np(targets) >= 0
    hot[ok, targets.cpu().numpy()[ok]] = scale * c
    off = 2.0 ** -13 * (np.abs(rd + hot) + np.abs(rd))
    lo, hi = (to_np(torch.from_numpy(rd + s * off).to(dtype)) for s in (-1, 1))
    got = to_np(logits.grad)
    assert np.all((lo <= got) & (got <= hi))
    assert abs(float(loss.detach()) - scale * rl.sum()) <= 1e-5 * scale * np.abs(rl).sum()
