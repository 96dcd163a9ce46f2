"""Float64 CPU oracle for causal attention with grouped heads over packed sequences.

TEST INFRASTRUCTURE ONLY, sharing no code with the HIP path. Per sequence s (queries cu_q[s] .. cu_q[s+1],
keys cu_k[s] .. cu_k[s+1]) and query head h, whose key head is h // (H // Hk), the plain definition on
whole score matrices: query i sees keys 0 .. i + Lk - Lq, a query without keys has out = 0 and lse = -inf.

    S = scale Q K^T;  P = exp(S - lse) on visible pairs, 0 elsewhere;  out = P V
    dV = P^T dO;  dP = dO V^T;  dS = P * (dP - rowsum(dO * out));  dQ = scale dS K;  dK = scale dS^T Q

with dK and dV summed over the query heads of a key head.

``bounds`` gives, element by element, how far a kernel may be off that holds its sums in 32 bits and
rounds to bf16 only P and dS before their products, out before Delta = rowsum(dO * out), and the results: a
rounding is off by at most u = 2^-8 of the value, so

    out   u (P |V| + |out|)
    Delta sum_d |dO| (out's bound)
    dV    u (P^T |dO| + |dV|)
    dQ    scale ((u |dS| + P Delta's bound) |K|) + u |dQ|       and dK likewise with |Q|
    lse   n 2^-24 scale |q| |k| for the n-term sums, and 2^-20 for exp and log in 32 bits

The 32-bit sums of n terms (D, and up to the keys or queries of the sequence) add n 2^-24 of the
magnitudes, which multiplies the bounds by at most 1 + 2^-2 for the n up to 2^14 used with them.
"""
from __future__ import annotations

import numpy as np

U = 2.0 ** -8


def causal_attention(q, k, v, dout, cu_q, cu_k, scale):
    """q, dout [Tq, H, D], k, v [Tk, Hk, D] as float arrays; dout None: forward only. Returns a dict of
    out, lse (and dq, dk, dv) in float64 and, under "bounds", their bounds."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    (Tq, H, D), (Tk, Hk) = q.shape, k.shape[:2]
    group = H // Hk
    out, lse = np.zeros((Tq, H, D)), np.full((H, Tq), -np.inf)
    b_out, b_lse = np.zeros((Tq, H, D)), np.zeros((H, Tq))
    back = dout is not None
    if back:
        dout = np.asarray(dout, dtype=np.float64)
        dq, dk, dv = np.zeros((Tq, H, D)), np.zeros((Tk, Hk, D)), np.zeros((Tk, Hk, D))
        b_dq, b_dk, b_dv = np.zeros((Tq, H, D)), np.zeros((Tk, Hk, D)), np.zeros((Tk, Hk, D))
    slack = 1.25
    for s in range(len(cu_q) - 1):
        a, b, c, d = int(cu_q[s]), int(cu_q[s + 1]), int(cu_k[s]), int(cu_k[s + 1])
        if a == b or c == d:
            continue
        sees = np.arange(d - c)[None] <= np.arange(b - a)[:, None] + (d - c) - (b - a)
        some = sees.any(1)
        for h in range(H):
            Q, K, V = q[a:b, h], k[c:d, h // group], v[c:d, h // group]
            S = np.where(sees, scale * (Q @ K.T), -np.inf)
            m = np.where(some, S.max(1), 0.0)
            E = np.exp(S - m[:, None])
            l = E.sum(1)
            P = E / np.where(some, l, 1.0)[:, None]
            o = P @ V
            out[a:b, h] = o
            with np.errstate(divide="ignore"):
                lse[h, a:b] = np.where(some, m + np.log(l), -np.inf)
            bo = slack * U * (P @ np.abs(V) + np.abs(o))
            b_out[a:b, h] = bo
            b_lse[h, a:b] = 2.0 ** -20 + D * 2.0 ** -24 * abs(scale) * (np.abs(Q) @ np.abs(K).T).max(1) \
                + 2.0 ** -22 * np.where(some, np.abs(m), 0.0)
            if not back:
                continue
            G = dout[a:b, h]
            dS = P * (G @ V.T - (G * o).sum(1)[:, None])
            dq[a:b, h] = scale * (dS @ K)
            dk[c:d, h // group] += scale * (dS.T @ Q)
            dv[c:d, h // group] += P.T @ G
            bS = U * np.abs(dS) + P * (np.abs(G) * bo).sum(1)[:, None]
            b_dq[a:b, h] = slack * (abs(scale) * (bS @ np.abs(K)) + U * np.abs(dq[a:b, h]))
            b_dk[c:d, h // group] += slack * abs(scale) * (bS.T @ np.abs(Q))
            b_dv[c:d, h // group] += slack * U * (P.T @ np.abs(G))
    res = {"out": out, "lse": lse, "bounds": {"out": b_out, "lse": b_lse}}
    if back:
        res.update(dq=dq, dk=dk, dv=dv)
        res["bounds"].update(dq=b_dq, dk=b_dk + slack * U * np.abs(dk), dv=b_dv + slack * U * np.abs(dv))
    return res
