"""Plain NumPy forms, in 64 bits, of the operators that a training step runs
around the scan: the convolution over a span, the embedding, the cross entropy
and the global gradient norm, each with its gradient. Test infrastructure only."""
import numpy as np


def _f64(a):
    return None if a is None else np.asarray(a, dtype=np.float64)


def _sigmoid(p):
    e = np.exp(-np.abs(p))
    return np.where(p >= 0, 1.0, e) / (1.0 + e)


def _taps(x, state):
    x = _f64(x)
    before = np.zeros((x.shape[0], 3, x.shape[2])) if state is None else _f64(state)
    return np.concatenate([before, x], axis=1)


def conv1d_pre(x, w, bias=None, state=None):
    """p [batch, L, width] (before SiLU) and sum of the magnitudes of its terms."""
    u, w = _taps(x, state), _f64(w)
    L = u.shape[1] - 3
    b = np.zeros(u.shape[2]) if bias is None else _f64(bias)
    p, mag = np.zeros(np.shape(x)) + b, np.zeros(np.shape(x)) + np.abs(b)
    for k in range(4):
        p += w[:, k] * u[:, k:k + L]
        mag += np.abs(w[:, k] * u[:, k:k + L])
    return p, mag


def conv1d(x, w, bias=None, state=None):
    """(out [batch, L, width], window after the span [batch, 3, width])."""
    p, _ = conv1d_pre(x, w, bias, state)
    return p * _sigmoid(p), _taps(x, state)[:, -3:]


def conv1d_backward(x, w, dout, bias=None, state=None, dstate_out=None):
    """dict(dx, dstate, dw, dbias, g): gradients, and g = dJ/dp."""
    u, w = _taps(x, state), _f64(w)
    L = u.shape[1] - 3
    p, _ = conv1d_pre(x, w, bias, state)
    s = _sigmoid(p)
    g = _f64(dout) * s * (1.0 + p * (1.0 - s))
    du = np.zeros_like(u)
    if dstate_out is not None:
        du[:, L:] += _f64(dstate_out)
    dw = np.zeros_like(w)
    for k in range(4):
        du[:, k:k + L] += w[:, k] * g
        dw[:, k] = np.sum(g * u[:, k:k + L], axis=(0, 1))
    return dict(dx=du[:, 3:], dstate=du[:, :3], dw=dw, dbias=np.sum(g, axis=(0, 1)), g=g)


def _valid(tokens, vocab):
    t = np.asarray(tokens).astype(np.int64)
    ok = (t >= 0) & (t < vocab)
    return t, ok


def embed(tokens, table, scale=1.0):
    """scale * table[tokens]; zeros for tokens outside the table."""
    table = _f64(table)
    t, ok = _valid(tokens, table.shape[0])
    out = np.zeros(t.shape + table.shape[1:])
    out[ok] = scale * table[t[ok]]
    return out


def embed_backward(tokens, dout, vocab, scale=1.0):
    """scale * sum of the rows of dout of each token."""
    t, ok = _valid(tokens, vocab)
    d = np.zeros((vocab, np.shape(dout)[-1]))
    np.add.at(d, t[ok], scale * _f64(dout)[ok])
    return d


def cross_entropy(logits, targets, weight=None, scale=1.0):
    """(loss, dlogits): weight * -log softmax(logits)[target] and its gradient
    times scale; zeros where the weight is zero or the target outside."""
    l = _f64(logits)
    n, V = l.shape
    t, ok = _valid(targets, V)
    w = np.ones(n) if weight is None else _f64(weight)
    ok = ok & (w != 0)
    loss, d = np.zeros(n), np.zeros((n, V))
    for i in np.nonzero(ok)[0]:
        m = np.max(l[i])
        e = np.exp(l[i] - m)
        loss[i] = w[i] * ((m - l[i, t[i]]) + np.log(np.sum(e)))   # m may be of the type's largest magnitude
        d[i] = e / np.sum(e)
        d[i, t[i]] -= 1.0
        d[i] *= w[i] * scale
    return loss, d


def grad_norm(tensors):
    return float(np.sqrt(sum(float(np.sum(_f64(t) ** 2)) for t in tensors)))


def clip_factor(norm, max_norm):
    return max_norm / norm if max_norm < norm < np.inf else 1.0
