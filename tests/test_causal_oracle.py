"""The causal oracle on the CPU: closed forms, torch's attention in float64 with autograd, differences, and
planted mistakes that these must catch."""
import importlib
import inspect

import numpy as np
import pytest
import torch

import oracle
mod = importlib.import_module("oracle.causal_attention")  # the module, which the function of its name hides


def _pack(lq, lk, H, Hk, D, seed=0):
    r = np.random.default_rng(seed)
    cu = lambda x: np.concatenate([[0], np.cumsum(x)]).astype(np.int32)  # noqa: E731
    tq, tk = sum(lq), sum(lk)
    return (r.standard_normal((tq, H, D)), r.standard_normal((tk, Hk, D)), r.standard_normal((tk, Hk, D)),
            r.standard_normal((tq, H, D)), cu(lq), cu(lk))


def _torch(q, k, v, dout, cu_q, cu_k, scale):
    q, k, v = (torch.tensor(x, requires_grad=True) for x in (q, k, v))
    g = q.shape[1] // k.shape[1]
    out = []
    for s in range(len(cu_q) - 1):
        Q = q[cu_q[s]:cu_q[s + 1]].transpose(0, 1)
        K, V = (x[cu_k[s]:cu_k[s + 1]].transpose(0, 1).repeat_interleave(g, 0) for x in (k, v))
        lq, lk = Q.shape[1], K.shape[1]
        mask = torch.ones(lq, lk, dtype=torch.bool).tril(lk - lq)
        some = mask.any(1)
        o = torch.nn.functional.scaled_dot_product_attention(Q, K, V, mask | ~some[:, None], scale=scale)
        out.append((o * some[:, None]).transpose(0, 1))
    out = torch.cat(out)
    out.backward(torch.tensor(dout))
    return [x.detach().numpy() for x in (out, q.grad, k.grad, v.grad)]


CASES = [([5, 1, 9], [5, 1, 9], 4, 2, 8), ([3, 1, 4], [7, 6, 4], 6, 2, 4), ([6, 3], [2, 3], 3, 1, 4)]


def _error(fn, case):
    p = _pack(*case)
    ref = _torch(*p, 0.3)
    got = fn(*p, 0.3)
    return max(np.abs(got[n] - r).max() for n, r in zip(("out", "dq", "dk", "dv"), ref))


@pytest.mark.parametrize("case", CASES)
def test_against_torch(case):
    assert _error(oracle.causal_attention, case) < 1e-10


def test_gradients_by_differences():
    q, k, v, g, cq, ck = _pack([4, 2], [5, 3], 4, 2, 4, seed=1)
    ref = oracle.causal_attention(q, k, v, g, cq, ck, 0.5)
    r = np.random.default_rng(2)
    for x, name in ((q, "dq"), (k, "dk"), (v, "dv")):
        d = r.standard_normal(x.shape)
        f = []
        for sign in (1, -1):
            y = {"dq": q, "dk": k, "dv": v}
            y[name] = x + sign * 1e-6 * d
            f.append((oracle.causal_attention(y["dq"], y["dk"], y["dv"], None, cq, ck, 0.5)["out"] * g).sum())
        assert abs((f[0] - f[1]) / 2e-6 - (ref[name] * d).sum()) < 1e-6


def test_first_token_and_rows_without_keys():
    q, k, v, g, cq, ck = _pack([3, 4], [3, 2], 2, 1, 4, seed=3)
    r = oracle.causal_attention(q, k, v, g, cq, ck, 0.7)
    assert np.allclose(r["out"][0], v[0]) and np.allclose(r["lse"][:, 0], 0.7 * (q[0] @ k[0, 0]))
    assert (r["out"][3:5] == 0).all() and np.isneginf(r["lse"][:, 3:5]).all() and (r["dq"][3:5] == 0).all()
    assert np.allclose(r["out"][5], v[3])  # the second sequence's third query sees its first key
    e = oracle.causal_attention(q, k[:0], v[:0], g, cq, [0, 0, 0], 0.7)
    assert (e["out"] == 0).all() and e["dk"].shape == (0, 1, 4)


MISTAKES = [("(d - c) - (b - a)", "0"), ("k[c:d, h // group]", "k[c:d, h % Hk]"), ("dk[c:d, h // group] +=", "dk[c:d, h // group] ="),
            ("dv[c:d, h // group] +=", "dv[c:d, h // group] ="), ("scale * (dS.T @ Q)", "dS.T @ Q"),
            ("(G * o).sum(1)", "(G * V[:1]).sum(1)"), ("<= np.arange", "< np.arange")]


@pytest.mark.parametrize("mistake", MISTAKES)
def test_planted_mistakes_are_caught(mistake):
    src = inspect.getsource(mod)
    assert src.count(mistake[0]) >= 1
    ns = {}
    exec(compile(src.replace(mistake[0], mistake[1]).replace("from __future__ import annotations", ""), "m", "exec"), ns)
    worst = 0.0
    for case in CASES:
        with np.errstate(all="ignore"):
            e = _error(ns["causal_attention"], case)
        worst = max(worst, np.inf if np.isnan(e) else e)
    assert worst > 1e-3
