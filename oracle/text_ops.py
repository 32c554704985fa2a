"""CPU oracle for the token table, the RMS normalisation with the residual's addition, rows in 8 bits and their product.
TEST INFRASTRUCTURE ONLY: it shares nothing with the HIP path and never imports it.

The paper's text encoder is a GPT-like Transformer (implementation details of the video-language model); its table and its norms
are standard and the paper writes no formula for them.  In fp64, one numpy expression per line of the definition:

    embedding :  y_i = s W[t_i], zeros for t_i outside [0, V);   dW[v] = s sum_{i: t_i = v} dy_i
    norm      :  rstd = 1 / sqrt(mean(h^2) + eps),  y = h rstd w        (h = x + residual, rounded by the caller)
                 dw = sum_rows dy xhat,  dh = rstd (g - xhat mean(g xhat)) + dh_in,   xhat = h rstd, g = dy w
    8 bits    :  scale = max(max|y|, 2^-96) / 448,  q = nearest e4m3 value of y / scale (ties to even)
    product   :  y_mn = sx_m sw_n sum_k x_mk w_nk + b_n
"""
from __future__ import annotations

import numpy as np

LEAST = 2.0 ** -96
E4M3_MAX = 448.0


def embedding_fwd(tokens, table, scale):
    t = np.asarray(tokens).reshape(-1)
    y = np.zeros((t.size, table.shape[1]))
    ok = (t >= 0) & (t < table.shape[0])
    y[ok] = np.asarray(table, dtype=np.float64)[t[ok]] * scale
    return y


def embedding_bwd(tokens, dy, V, scale):
    """dW [V, D], and the sum of magnitudes behind each of its elements."""
    t = np.asarray(tokens).reshape(-1)
    dy = np.asarray(dy, dtype=np.float64).reshape(t.size, -1)
    ok = (t >= 0) & (t < V)
    dw, mag = np.zeros((V, dy.shape[1])), np.zeros((V, dy.shape[1]))
    np.add.at(dw, t[ok], dy[ok])
    np.add.at(mag, t[ok], np.abs(dy[ok]))
    return dw * scale, mag * abs(scale)


def rms_fwd(h, w, eps):
    """y [M, D], rstd [M]."""
    h = np.asarray(h, dtype=np.float64)
    rstd = 1.0 / np.sqrt((h * h).mean(axis=1) + eps)
    return h * rstd[:, None] * np.asarray(w, dtype=np.float64), rstd


def rms_bwd(h, w, dy, dh, eps):
    """dh (of h, so of x and of the residual), dw."""
    h, w, dy = (np.asarray(a, dtype=np.float64) for a in (h, w, dy))
    rstd = (1.0 / np.sqrt((h * h).mean(axis=1) + eps))[:, None]
    xhat, g = h * rstd, dy * w
    d = rstd * (g - xhat * (g * xhat).mean(axis=1, keepdims=True))
    return d + (0.0 if dh is None else np.asarray(dh, dtype=np.float64)), (dy * xhat).sum(axis=0)


def e4m3_values():
    """The finite non-negative values of the format, from its definition: 3 bits of fraction, exponent bias 7, 0x7f is NaN."""
    v = []
    for code in range(0x7f):
        e, f = code >> 3, code & 7
        v.append(f * 2.0 ** -9 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7))
    return np.array(v)


def e4m3_half_step(v):
    """Half the distance of the format's values around |v| (of the binade that |v| lies in)."""
    a = np.maximum(np.abs(np.asarray(v, dtype=np.float64)), 2.0 ** -6)
    return 2.0 ** (np.floor(np.log2(a)) - 4)


def e4m3(v):
    """Nearest value of the format by search among all of them; ties to the even code."""
    vals, a = e4m3_values(), np.abs(np.asarray(v, dtype=np.float64))
    hi = np.clip(np.searchsorted(vals, a), 1, vals.size - 1)
    lo = hi - 1
    up = vals[hi] - a < a - vals[lo]
    tie = vals[hi] - a == a - vals[lo]
    code = np.where(up | (tie & (hi % 2 == 0)), hi, lo)
    return np.copysign(vals[code], v)


def rows8(y):
    """q [M, D] (values), scale [M]."""
    y = np.asarray(y, dtype=np.float64)
    scale = np.maximum(np.abs(y).max(axis=1), LEAST) / E4M3_MAX
    return e4m3(y / scale[:, None]), scale


def linear(x, sx, w, sw, b):
    """y [M, N], and the sum of magnitudes behind each element's contraction."""
    x, sx, w, sw = (np.asarray(a, dtype=np.float64) for a in (x, sx, w, sw))
    s = sx[:, None] * sw
    return (x @ w.T) * s + (0.0 if b is None else np.asarray(b, dtype=np.float64)), (np.abs(x) @ np.abs(w).T) * np.abs(s)
