"""The operators of decoding in 8 bits and of drawing tokens, from their definitions, in 64 bits (numpy). Used by the tests
and the smoke check only; shares no code with the library."""
import numpy as np

BLOCK = 128


def stride(width):
    """Bytes of a row of scales."""
    return 4 * -(-width // (4 * BLOCK))


def e4m3_values(q):
    """Bytes as e4m3 numbers: sign, 4 exponent bits (bias 7), 3 of the mantissa; 0x7f is NaN."""
    q = np.asarray(q, np.uint8).astype(np.int64)
    e, m = q >> 3 & 15, q & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (np.maximum(e, 1) - 10.0))
    v = np.where((q & 127) == 127, np.nan, v)
    return np.where(q >> 7 == 1, -v, v)


def e4m3_round(x):
    """x to the nearest e4m3 number, ties to even; |x| <= 448 (NaN stays)."""
    a = np.abs(x)
    with np.errstate(divide="ignore"):
        e = np.floor(np.log2(np.where(a > 0, a, 1.0)))
    e = np.where(a < 2.0 ** e, e - 1, np.where(a >= 2.0 ** (e + 1), e + 1, e))   # log2 may round over a power of two
    step = 2.0 ** (np.maximum(e, -6) - 3)
    return np.rint(x / step) * step


def block_exponent(top):
    """The smallest E >= -126 with top <= 448 2^E; 0 for 0."""
    if top == 0:
        return 0
    e = int(np.ceil(np.log2(top / 448.0))) - 1
    while top > 448.0 * 2.0 ** e:
        e += 1
    return max(e, -126)


def quantize(x, block_rows):
    """x [rows, width] -> values (before scaling) and scale bytes [ceil(rows / block_rows), stride]."""
    x = np.asarray(x, np.float64)
    rows, width = x.shape
    q = np.empty_like(x)
    scales = np.full((-(-rows // block_rows), stride(width)), 127, np.uint8)
    finite = np.isfinite(x)
    for i in range(0, rows, block_rows):
        for j in range(0, width, BLOCK):
            at = np.s_[i:i + block_rows, j:j + BLOCK]
            e = block_exponent(np.max(np.abs(x[at]), where=finite[at], initial=0.0))
            q[at] = np.where(finite[at], e4m3_round(np.where(finite[at], x[at], 0.0) * 2.0 ** -e), np.nan)
            scales[i // block_rows, j // BLOCK] = e + 127
    return q, scales


def factors(scales, block_rows, rows, width):
    """Scale bytes as a factor for each element."""
    f = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return np.repeat(np.repeat(f, block_rows, 0)[:rows], BLOCK, 1)[:, :width]


def dequantize(q, scales, block_rows):
    """Bytes and scale bytes -> the values they stand for."""
    return e4m3_values(q) * factors(scales, block_rows, *q.shape)


def rmsnorm(residual, w, eps):
    return residual * w / np.sqrt(np.mean(residual * residual, 1, keepdims=True) + eps)


def matmul(a, a_scales, w, w_scales):
    """The product, and the same of magnitudes (what rounding errors are relative to)."""
    x, y = dequantize(a, a_scales, 1), dequantize(w, w_scales, BLOCK)
    return x @ y.T, np.abs(x) @ np.abs(y).T


def kept(logits, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, most=np.finfo(np.float32).max):
    """One row: weights of the tokens that may be drawn (0 for the others), by index."""
    l = np.minimum(np.where(np.isnan(logits), -np.inf, np.asarray(logits, np.float64)), most)
    n = l.size
    order = sorted((i for i in range(n) if l[i] > -np.inf), key=lambda i: (-l[i], i))
    w = np.zeros(n)
    if not order:
        return w
    if not temperature > 0:
        w[order[0]] = 1.0
        return w
    if 0 < top_k < n:
        order = order[:top_k]
    weight = {i: float(np.exp((l[i] - l[order[0]]) / temperature)) for i in order}
    total, before, keep = sum(weight.values()), 0.0, []
    for i in order:
        if keep and top_p < 1 and before >= top_p * total:
            break
        keep.append(i)
        before += weight[i]
    for i in keep:
        if not (min_p > 0 and weight[i] < min(min_p, 1.0)):
            w[i] = weight[i]
    return w


def sample(logits, u, **settings):
    """One row: (token, its probability)."""
    w = kept(logits, **settings)
    if not w.any():
        return -1, 0.0
    upto = np.cumsum(w)
    u = 0.0 if not u > 0 else u
    at = int(np.searchsorted(upto, u * upto[-1], side="right"))
    if at >= w.size or w[at] == 0:   # u of 1 or more
        at = int(np.nonzero(w)[0][-1])
    return at, float(w[at] / upto[-1])
