"""The sequence layers in 64 bits, from their definitions (include/wpk.h), with the normalisers their tolerances need.

Everything is NumPy float64, token by token; requests are (start, length) pairs and states are per request."""
import numpy as np
from math import erf

_erf = np.vectorize(erf, otypes=[np.float64])


def act(v, name):
    if name == "relu":
        return np.maximum(v, 0.0)
    if name == "silu":
        with np.errstate(over="ignore"):
            return v / (1.0 + np.exp(-v))
    if name == "gelu":
        return 0.5 * v * (1.0 + _erf(v * np.sqrt(0.5)))
    return v


def linear(x, w, bias=None, residual=None, act_name="none"):
    """(y, sum of the magnitudes that y is summed from)."""
    v, d = x @ w.T, np.abs(x) @ np.abs(w).T
    if bias is not None:
        v, d = v + bias, d + np.abs(bias)
    v = act(v, act_name)
    if residual is not None:
        v, d = v + residual, d + np.abs(residual)
    return v, d


def causal_conv1d(x, w, bias, rows, history, act_name="silu"):
    """x [tokens][channels]; rows: (start, length) of every request; history: [width-1][channels] of every request.
    Returns (y, magnitudes, new history of every request); rows of no request are NaN."""
    past = w.shape[1] - 1
    y, d = np.full(x.shape, np.nan), np.zeros(x.shape)
    left = []
    for (a, n), h in zip(rows, history):
        line = np.concatenate([h, x[a:a + n]])
        for t in range(n):
            terms = line[t:t + past + 1].T * w
            v = terms.sum(1) + (0.0 if bias is None else bias)
            d[a + t] = np.abs(terms).sum(1) + (0.0 if bias is None else np.abs(bias))
            y[a + t] = act(v, act_name)
        left.append(line[n:])
    return y, d, left


def ssm_scan(x, dt, a, b, c, rows, state, d_skip=None, z=None, dt_bias=None, softplus=True):
    """x, z [tokens][heads][head_dim], dt [tokens][heads], b, c [tokens][groups][state_dim]; state: [heads][head_dim][state_dim]
    of every request.  Returns (y, magnitudes of y, new states, magnitudes of the states)."""
    heads, groups = x.shape[1], b.shape[1]
    of = np.arange(heads) // (heads // groups)
    y, dy = np.full(x.shape, np.nan), np.zeros(x.shape)
    left, dleft = [], []
    for (t0, n), h in zip(rows, state):
        h, m = h.copy(), np.abs(h)
        for t in range(t0, t0 + n):
            delta = dt[t] + (0.0 if dt_bias is None else dt_bias)
            if softplus:
                delta = np.logaddexp(0.0, delta)
            keep = np.exp(delta * a)[:, None, None]
            feed = (delta[:, None] * x[t])[:, :, None] * b[t][of][:, None, :]
            h, m = keep * h + feed, keep * m + np.abs(feed)
            v, s = np.einsum("hpn,hn->hp", h, c[t][of]), np.einsum("hpn,hn->hp", m, np.abs(c[t][of]))
            if d_skip is not None:
                v, s = v + d_skip[:, None] * x[t], s + np.abs(d_skip[:, None] * x[t])
            if z is not None:
                g = act(z[t], "silu")
                v, s = v * g, s * np.abs(g)
            y[t], dy[t] = v, s
        left.append(h)
        dleft.append(m)
    return y, dy, left, dleft
