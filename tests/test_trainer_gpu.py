"""The training example (trainer.py): its gradients against autograd over a
plain 64-bit model, and that its steps learn.

Bound: everything runs in fp32 (sums of up to a few hundred terms, the scan
within 1e-4 of the oracle by its own bar); errors pass through two layers, so a
gradient may be off by 1e-3 of its tensor's largest magnitude."""
import pytest
import torch

from paper_2401_13660_gb300.decoder import CONFIGS
from paper_2401_13660_gb300.trainer import Model, Trainer

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _plain_loss(model, params, tokens, targets, counted):
    """The same model in torch operations on 64-bit leaves (in model.parameters' order)."""
    cfg = model.cfg
    it = iter(params)
    layers = [{k: next(it) for k in L} for L in model.layers]
    emb, norm_f = next(it), next(it)
    R, N = cfg.dt_rank, cfg.d_state

    def norm(r, w):
        return r * torch.rsqrt(r.square().mean(-1, keepdim=True) + cfg.eps) * w
    ok = (tokens >= 0) & (tokens < cfg.vocab)
    res = emb[tokens.clamp(0, cfg.vocab - 1)] * ok[..., None] * cfg.d_model ** 0.5
    for L in layers:
        h = norm(res, L["norm_w"])
        x, z = h @ L["W_in"][0].t(), h @ L["W_in"][1].t()
        pad = torch.nn.functional.pad(x, (0, 0, 3, 0))
        xc = torch.nn.functional.silu(sum(pad[:, k:k + x.shape[1]] * L["conv_w"][:, k] for k in range(4)) + L["conv_b"])
        rows = xc @ L["W_xproj"].t()
        delta = torch.nn.functional.softplus(rows[..., :R] @ L["W_dt"].t() + L["dt_bias"])
        B, C = rows[..., R:R + N], rows[..., R + N:]
        s = torch.zeros(x.shape[0], x.shape[2], N, device=DEV, dtype=torch.float64)
        ys = []
        for t in range(x.shape[1]):
            s = torch.exp(delta[:, t, :, None] * L["A"]) * s + (delta[:, t] * xc[:, t])[..., None] * B[:, t, None]
            ys.append((s * C[:, t, None]).sum(-1) + L["D"] * xc[:, t])
        res = res + (torch.stack(ys, 1) * torch.nn.functional.silu(z)) @ L["W_out"].t()
    logp = torch.log_softmax(norm(res, norm_f) @ emb.t(), -1)
    hit = (targets >= 0) & (targets < cfg.vocab)
    return -(logp.gather(-1, targets.clamp(0, cfg.vocab - 1)[..., None])[..., 0] * hit).sum() / counted


def test_gradients_match_a_plain_64_bit_model():
    model = Model(CONFIGS["tiny_2x64"], DEV, dtype=torch.float32, seed=3)
    g = torch.Generator(device=DEV).manual_seed(1)
    tokens = torch.randint(0, 256, (3, 37), device=DEV, generator=g)
    targets = torch.randint(0, 256, (3, 37), device=DEV, generator=g)
    tokens[1, 30:], targets[1, 29:] = -1, -1   # a shorter row
    counted = int((targets >= 0).sum())
    loss = model.loss(tokens, targets, counted)
    loss.backward()
    model.check()
    wide = [p.detach().double().requires_grad_() for p in model.parameters]
    want = _plain_loss(model, wide, tokens, targets, counted)
    want.backward()
    assert abs(float(loss.detach()) - float(want.detach())) <= 1e-4 * float(want.detach())
    for p, q in zip(model.parameters, wide):
        assert float((p.grad.double() - q.grad).abs().max()) <= 1e-3 * float(q.grad.abs().max())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_steps_learn_and_are_clipped(dtype):
    model = Model(CONFIGS["tiny_2x64"], DEV, dtype=dtype, seed=0)
    trainer = Trainer(model, lr=3e-3, max_norm=0.5)
    row = torch.arange(97, 123, device=DEV, dtype=torch.uint8).repeat(2 * 6)[:2 * 130].view(2, 130)
    first = last = None
    for _ in range(40):
        loss, norm = trainer.train_step(row[:, :-1].contiguous(), row[:, 1:].contiguous())
        first = float(loss) if first is None else first
        last = float(loss)
        total = sum(float(t.double().square().sum()) for t in trainer.grads.tensors) ** 0.5
        assert total <= min(0.5, float(norm)) * (1 + 2.0 ** -7)
    model.check()
    assert first > 5.0 and last < 0.5 * first


def test_the_example_runs(capsys, monkeypatch):
    from paper_2401_13660_gb300 import trainer
    monkeypatch.setattr("sys.argv", ["trainer", "--steps", "6", "--length", "64", "--batch", "2"])
    trainer.main()
    lines = capsys.readouterr().out.splitlines()
    assert len(lines) == 2 and all("bits per byte" in line for line in lines)
