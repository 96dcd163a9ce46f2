"""Float64 CPU oracle for norms of heads with rotary positions after them, forward and backward.

TEST INFRASTRUCTURE ONLY, sharing no code with the HIP path. x [T, H, D]; per token and head

    x^ = x r,  r = 1 / sqrt(mean(x^2) + eps);  n = w x^;  y = R n
    dn = R^T dy;  dw = sum_{t, h} dn x^;  dx = r (w dn - x^ mean(w dn x^))

with R the turn of the first 2 n dimensions by position * frequency (times mscale), the others kept.

Each result comes with how far a kernel may be off that computes in 32 bits and rounds the result to bf16 once. A rounding
to 32 bits is off by at most e = 2^-24 of the value, one to bf16 by 2^-8. The norm: at most 25 roundings in the mean of squares,
whose error the root halves, 4 e of the reciprocal root, two products and r's own: under 32 e = 2^-19 of x^ and n. The turn: sine and
cosine off by 2^-22, two products and a sum: 2^-21 mscale (|a| + |b|) of a pair (a, b). The backward pass's row sum has 25
roundings as the norm's, its other steps three. A term of dw's sums is rounded as often as weight_depth says.
"""
from __future__ import annotations

import numpy as np

E = 2.0 ** -24
NORM, TURN = 32 * E, 8 * E


def _pairs(n, layout):
    return (slice(0, n), slice(n, 2 * n)) if layout == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))


def turned(x, err, positions, freqs, layout, sections, mscale, sign=1.0):
    """R x (or its transpose, sign -1) and its error, given x's. positions int [axes, T] or None (no turn)."""
    if freqs is None:
        return x, err
    axis = np.repeat(np.arange(len(sections)), sections)
    angle = np.asarray(positions).reshape(len(sections), -1)[axis].T.astype(np.longdouble) * np.asarray(freqs, dtype=np.longdouble)
    angle = np.asarray(np.mod(angle, np.longdouble("6.28318530717958647692528676655900577")), dtype=np.float64)
    c, s = np.cos(angle)[:, None] * mscale, sign * np.sin(angle)[:, None] * mscale
    a, b = _pairs(len(freqs), layout)
    y, e = x.copy(), np.array(err, copy=True)
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    own = TURN * abs(mscale) * (np.abs(x[..., a]) + np.abs(x[..., b]))
    e[..., a], e[..., b] = (np.abs(c) * err[..., a] + np.abs(s) * err[..., b] + own,
                            np.abs(s) * err[..., a] + np.abs(c) * err[..., b] + own)
    return y, e


def forward(x, w, eps, *turn):
    """y and its bound. turn: positions, freqs, layout, sections, mscale."""
    x = np.asarray(x, dtype=np.float64)
    n = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * (1.0 if w is None else np.asarray(w, dtype=np.float64))
    y, e = turned(n, NORM * np.abs(n), *turn)
    return y, e + 2.0 ** -8 * np.abs(y)


def weight_depth(T, H, D):
    """Sums that a term of dw goes through: those of a lane, which adds up its rows one after the other, of the 4096 / D groups of lanes of a workgroup, and of the
    workgroups (two by a thread, eight steps of a tree). A workgroup has at most T / 256 tokens; its groups share the rows of eight or more of them at a time."""
    groups, tokens = 4096 // D, -(-T // 256)
    return -(-tokens * H // groups) + tokens // 8 + 2 + groups + 2 + 8


def backward(x, dy, w, eps, *turn, weight_step=0.0):
    """dx, dw and their bounds; weight_step: the rounding of dw (2^-8 for bf16)."""
    x, dy = np.asarray(x, dtype=np.float64), np.asarray(dy, dtype=np.float64)
    w = np.ones(x.shape[-1]) if w is None else np.asarray(w, dtype=np.float64)
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    xhat = x * r
    dn, e_dn = turned(dy, np.zeros_like(dy), *turn, sign=-1.0)
    g, e_g = w * dn, np.abs(w) * e_dn
    c = (g * xhat).mean(-1, keepdims=True)
    e_c = (e_g * np.abs(xhat) + (NORM + 25 * E) * np.abs(g * xhat)).mean(-1, keepdims=True)
    dx = r * (g - xhat * c)
    e_dx = r * (e_g + np.abs(xhat) * e_c + 2 * NORM * (np.abs(g) + np.abs(xhat * c))) + 2.0 ** -8 * np.abs(dx)
    dw = (dn * xhat).sum((0, 1))
    e_dw = (e_dn * np.abs(xhat) + (NORM + weight_depth(*x.shape) * E) * np.abs(dn * xhat)).sum((0, 1)) + weight_step * np.abs(dw)
    return dx, dw, e_dx, e_dw
