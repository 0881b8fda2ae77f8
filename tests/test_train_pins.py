"""The 64-bit forms in oracle/train.py against central differences, against
step-by-step decoding and against sums written out (CPU)."""
import numpy as np
import pytest

import oracle
from oracle import train


def _differences(f, a, eps=1e-6):
    """dJ/da of the scalar function f by central differences, entry by entry."""
    d = np.zeros_like(a)
    for i in np.ndindex(a.shape):
        keep = a[i]
        a[i] = keep + eps
        up = f()
        a[i] = keep - eps
        d[i] = (up - f()) / (2 * eps)
        a[i] = keep
    return d


@pytest.mark.parametrize("b, L, D", [(1, 1, 2), (2, 2, 3), (1, 3, 2), (2, 7, 3)])
def test_conv_gradients_are_the_differences(b, L, D):
    g = np.random.default_rng(L)
    x, w, bias, state = g.normal(size=(b, L, D)), g.normal(size=(D, 4)), g.normal(size=D), g.normal(size=(b, 3, D))
    dout, dso = g.normal(size=(b, L, D)), g.normal(size=(b, 3, D))

    def J():
        out, so = train.conv1d(x, w, bias, state)
        return np.sum(out * dout) + np.sum(so * dso)
    got = train.conv1d_backward(x, w, dout, bias, state, dso)
    for name, a in (("dx", x), ("dw", w), ("dbias", bias), ("dstate", state)):
        # truncation 1e-12 |J'''|, rounding 1e-16 |J| / 1e-6
        np.testing.assert_allclose(got[name], _differences(J, a), rtol=1e-7, atol=1e-7)


@pytest.mark.parametrize("L", [1, 2, 3, 9])
def test_conv_is_its_steps(L):
    g = np.random.default_rng(L)
    x, w, bias, state = g.normal(size=(2, L, 5)), g.normal(size=(5, 4)), g.normal(size=5), g.normal(size=(2, 3, 5))
    out, so = train.conv1d(x, w, bias, state)
    for t in range(L):
        o, state = oracle.conv1d_step(state, x[:, t], w, bias)
        np.testing.assert_allclose(out[:, t], o, rtol=1e-13, atol=1e-13)
    np.testing.assert_array_equal(so, state)


def test_embedding_gradient_is_the_differences():
    g = np.random.default_rng(0)
    tokens, table, dout = np.array([3, 0, -1, 3, 7, 4]), g.normal(size=(5, 2)), g.normal(size=(6, 2))
    d = _differences(lambda: np.sum(train.embed(tokens, table, 1.7) * dout), table)
    np.testing.assert_allclose(train.embed_backward(tokens, dout, 5, 1.7), d, rtol=1e-8, atol=1e-8)


def test_cross_entropy_gradient_is_the_differences():
    g = np.random.default_rng(1)
    logits, weight = g.normal(size=(5, 4)), np.array([1.0, 0.5, 0.0, 2.0, 1.0])
    targets = np.array([0, 3, 1, -1, 2])
    loss, dl = train.cross_entropy(logits, targets, weight, 0.25)
    assert loss[2] == 0 and loss[3] == 0 and not dl[2].any() and not dl[3].any()
    d = _differences(lambda: 0.25 * np.sum(train.cross_entropy(logits, targets, weight)[0]), logits)
    np.testing.assert_allclose(dl, d, rtol=1e-7, atol=1e-8)
    p = np.exp(logits[0]) / np.sum(np.exp(logits[0]))
    np.testing.assert_allclose(loss[0], -np.log(p[0]), rtol=1e-13)


def test_clip_factor():
    assert train.grad_norm([np.array([3.0]), np.array([[0.0, 4.0]])]) == 5.0
    assert train.clip_factor(5.0, 1.0) == 0.2 and train.clip_factor(5.0, 5.0) == 1.0
    assert train.clip_factor(np.inf, 1.0) == 1.0 and train.clip_factor(np.nan, 1.0) == 1.0
