"""Steps of the training example (trainer.py) that must not change the model:
a device-side error, a norm that is not finite."""
import pytest
import torch

from paper_2401_13660_gb300 import mbscan as mb
from paper_2401_13660_gb300.decoder import CONFIGS
from paper_2401_13660_gb300.trainer import Model, Trainer

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _trainer(dtype=torch.bfloat16):
    model = Model(CONFIGS["tiny_2x64"], DEV, dtype=dtype, seed=5)
    return model, Trainer(model, lr=1e-2, max_norm=0.5)


def _rows(seed, L=40):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randint(0, 256, (2, L), device=DEV, generator=g)


def _state(trainer):
    """Copies of everything that a step changes."""
    opt = [v.clone() for p in trainer.model.parameters for _, v in sorted(trainer.optimizer.state.get(p, {}).items())]
    return [p.detach().clone() for p in trainer.model.parameters] + opt


def _same(a, b):
    return len(a) == len(b) and all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("L", [16, 400])   # the workspace stays, or grows within the step
def test_a_device_side_error_stops_the_step(L):
    model, trainer = _trainer()
    trainer.train_step(_rows(0, 16), _rows(1, 16))
    before = _state(trainer)
    mb.mb_selftest_timeout(model.ws.buffer, 100_000)   # a wait that ran out, as a scan would record it
    with pytest.raises(mb.MbError):
        trainer.train_step(_rows(2, L), _rows(3, L))
    assert _same(before, _state(trainer))
    trainer.train_step(_rows(2, L), _rows(3, L))       # read and cleared: steps go on
    assert not _same(before, _state(trainer))


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_norm_that_is_not_finite_skips_the_step(bad):
    model, trainer = _trainer()
    for i in range(2):
        trainer.train_step(_rows(i), _rows(i + 1))
    before = _state(trainer)
    with torch.no_grad():
        keep = model.layers[0]["D"][3].clone()
        model.layers[0]["D"][3] = bad
    _, norm = trainer.train_step(_rows(2), _rows(3))
    assert not torch.isfinite(norm).any()
    with torch.no_grad():
        model.layers[0]["D"][3] = keep
    assert _same(before, _state(trainer))              # weights, moments and step counts
    loss, norm = trainer.train_step(_rows(2), _rows(3))
    assert torch.isfinite(loss).all() and torch.isfinite(norm).all() and not _same(before, _state(trainer))
