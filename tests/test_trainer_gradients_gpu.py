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


def _function_calls():
    ws = tr.Workspace(DEV)
    g = torch.Generator(device=DEV).manual_seed(6)
    rnd = lambda *s: torch.randn(*s, device=DEV, generator=g)
    leaf = lambda *s: rnd(*s).requires_grad_()
    tokens = torch.randint(0, 256, (2, 20), device=DEV, generator=g)
    A = (-torch.rand(16, 16, device=DEV, generator=g) - 0.5).requires_grad_()
    return dict(
        Embed=lambda x: tr.Embed.apply(x, tokens, 2.0, ws),
        Conv1d=lambda x: tr.Conv1d.apply(x, leaf(16, 4), leaf(16), ws),
        Scan=lambda x: tr.Scan.apply(x, leaf(2, 20, 16), leaf(2, 20, 16), leaf(2, 20, 16), leaf(2, 20, 16), A, leaf(16), leaf(16), ws),
        CrossEntropy=lambda x: tr.CrossEntropy.apply(x, tokens, 0.1))


@pytest.mark.parametrize("name, shape", [("Embed", (256, 16)), ("Conv1d", (2, 20, 16)), ("Scan", (2, 20, 16)),
                                         ("CrossEntropy", (2, 20, 256))])
def test_a_second_derivative_is_an_error(name, shape):
    # the kernels give first derivatives only: a backward through a backward would drop what it leaves out
    x = torch.randn(*shape, device=DEV, generator=torch.Generator(device=DEV).manual_seed(7)).requires_grad_()
    out = (_function_calls()[name](x) ** 2).sum()
    (d,) = torch.autograd.grad(out, x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        d.square().sum().backward()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradient_of_the_tied_table_is_rounded_once(dtype, monkeypatch):
    # The head's part and the lookup's are fp32 sums of at most n terms each, joined before anything is rounded: the
    # gradient lies between the roundings of the ends of 2 (n + 4) u times the sum of the terms' magnitudes.
    from paper_2401_13660_gb300.decoder import CONFIGS
    model = tr.Model(CONFIGS["tiny_2x64"], DEV, dtype=dtype, seed=8)
    g = torch.Generator(device=DEV).manual_seed(9)
    tokens = torch.randint(0, 40, (2, 40), device=DEV, generator=g)
    tokens[1, 30:] = -1
    d = torch.randn(2, 40, 256, device=DEV, generator=g).to(dtype)
    douts, hs = [], []
    backward, norm = tr.mb.mb_embed_backward, tr.rmsnorm
    monkeypatch.setattr(tr.mb, "mb_embed_backward", lambda t, dout, *a, **k: (douts.append(dout.clone()), backward(t, dout, *a, **k))[1])
    monkeypatch.setattr(tr, "rmsnorm", lambda *a: (hs.append(norm(*a)), hs[-1])[1])
    logits = model.logits(tokens)
    t, dn, hn = tokens.cpu().numpy(), to_np(d).reshape(80, 256), to_np(hs[-1]).reshape(80, -1)
    scale = float(np.float32(model.cfg.d_model ** 0.5))
    for again in (True, False):   # twice through one graph (the scan's gradients have no fixed order: each by its own)
        model.emb.grad = None
        logits.backward(d, retain_graph=again)
        out, x = to_np(douts[-1]), to_np(model.emb.grad)
        ref = dn.T @ hn + train.embed_backward(t, out, 256, scale)
        off = 2 * (80 + 4) * 2.0 ** -24 * (np.abs(dn).T @ np.abs(hn) + train.embed_backward(t, np.abs(out), 256, scale))
        lo, hi = (to_np(torch.from_numpy(ref + s * off).to(dtype)) for s in (-1, 1))
        assert np.all((lo <= x) & (x <= hi)), float(np.mean((lo > x) | (x > hi)))
    assert len(douts) == 2
