"""What stands around a mixer layer in 64 bits, from the definitions (include/wpk.h): normalisation, 8-bit values, products in 8
bits and by expert, the router; with the magnitudes their tolerances need.

Everything is NumPy float64 but the 8-bit rounding, whose steps in 32 bits are part of its definition."""
import numpy as np

from oracle.sequence import act

BLOCK = 128
LARGEST = 448.0


def blocks(width):
    return -(-width // BLOCK)


def e4m3_values():
    """The number that each of the 256 codes stands for."""
    out = np.empty(256)
    for c in range(256):
        e, m = c >> 3 & 15, c & 7
        v = np.nan if e == 15 and m == 7 else (1 + m / 8) * 2.0 ** (e - 7) if e else m * 2.0 ** -9
        out[c] = -v if c & 128 else v
    return out


def round_e4m3(v):
    """The e4m3 number nearest to v, ties to the even mantissa, none beyond 448."""
    v = np.asarray(v, np.float64)
    with np.errstate(divide="ignore", invalid="ignore"):
        e = np.floor(np.log2(np.abs(v)))
        step = 2.0 ** (np.maximum(np.where(np.isfinite(e), e, -6), -6) - 3)
        return np.clip(np.round(v / step) * step, -LARGEST, LARGEST)


def quantize(v):
    """(q as numbers, scales) of float32 rows, by the definition's own steps in 32 bits."""
    v = np.asarray(v, np.float32)
    rows, width = v.shape
    q, scales = np.empty(v.shape), np.empty((rows, blocks(width)), np.float32)
    with np.errstate(invalid="ignore", over="ignore"):
        for b in range(blocks(width)):
            part = v[:, b * BLOCK:(b + 1) * BLOCK]
            most = np.fmax.reduce(np.abs(part), axis=1)
            s = np.fmax(most / np.float32(LARGEST), np.float32(2.0 ** -110))
            inverse = np.float32(1.0) / s
            q[:, b * BLOCK:(b + 1) * BLOCK] = round_e4m3(part * inverse[:, None])
            scales[:, b] = s
    return q, scales


def spread(scales, shape, rows=1):
    """Scales at every value: one for `rows` rows and a block of columns."""
    s = np.repeat(np.asarray(scales, np.float64), BLOCK, axis=1)[:, :shape[1]]
    return np.repeat(s, rows, axis=0)[:shape[0]]


def rms_norm(x, gain, eps, residual=None, groups=1, parts=1, source=None, weights=None):
    """(s, magnitudes of s, v): x [x_rows][width]."""
    rows = len(source) if source is not None else len(x) // parts
    s = np.zeros((rows, x.shape[1])) if residual is None else residual.copy()
    d = np.abs(s)
    for t in range(rows):
        for j in range(parts):
            r = t * parts + j if source is None else source[t][j]
            if 0 <= r < len(x):
                term = x[r] * (1.0 if weights is None else weights[t][j])
                s[t], d[t] = s[t] + term, d[t] + np.abs(term)
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        by = s.reshape(rows, groups, -1)
        v = (by / np.sqrt((by ** 2).mean(2, keepdims=True) + eps)).reshape(s.shape) * (1.0 if gain is None else gain)
    return s, d, v


def grouped(x, w, starts, source=None, act_name="none", gated=False):
    """(y, magnitudes, covered rows): w [groups][n or 2 n][k]; rows of no expert are NaN."""
    rows = starts[-1] if source is None else len(source)
    n = w.shape[1] // (2 if gated else 1)
    y, d = np.full((max(rows, len(x) if source is None else rows), n), np.nan), np.zeros((max(rows, len(x) if source is None else rows), n))
    for g in range(len(w)):
        a, b = starts[g], starts[g + 1]
        xs = x[a:b] if source is None else x[np.clip(source[a:b], 0, len(x) - 1)]
        v, m = xs @ w[g].T, np.abs(xs) @ np.abs(w[g]).T
        if gated:
            left, right = act(v[:, :n], act_name), v[:, n:]
            y[a:b], d[a:b] = left * right, m[:, :n] * np.abs(right) + (np.abs(left) + m[:, :n]) * m[:, n:]
        else:
            y[a:b], d[a:b] = act(v, act_name), m
    return y, d


def route(logits, k, normalize=True, scale=1.0):
    """(experts, weights, starts, source, place)."""
    tokens, n = logits.shape
    l = np.where(np.isnan(logits), -np.inf, logits) + 0.0
    experts = np.argsort(-l, axis=1, kind="stable")[:, :k]
    top = np.take_along_axis(l, experts, 1)
    with np.errstate(invalid="ignore"):
        e = np.exp(top - top[:, :1])
        total = e.sum(1) if normalize else np.exp(l - top[:, :1]).sum(1)
        weights = np.where(top[:, :1] == -np.inf, 0.0, scale * e / total[:, None])
    flat = experts.reshape(-1)
    order = np.argsort(flat, kind="stable")
    place = np.empty_like(order)
    place[order] = np.arange(order.size)
    starts = np.concatenate([[0], np.cumsum(np.bincount(flat, minlength=n))])
    return experts, weights, starts, order // k, place.reshape(tokens, k)
