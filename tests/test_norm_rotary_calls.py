"""Norms of heads with rotary positions, on the CPU: the oracle's gradients against differences, refusals by the C ABI (fake
addresses, never dereferenced) and by the binding."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2607_01701_amd as t2v
from oracle import norm_rotary as oracle
from paper_2607_01701_amd import _lib

from test_autograd_calls import HOOKS, calls  # noqa: F401

A, MB = 0x100000, 1 << 20
INV, UNS, WS = _lib.T2V_ERR_INVALID_ARG, _lib.T2V_ERR_UNSUPPORTED, _lib.T2V_ERR_WORKSPACE


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("weights", [True, False])
def test_oracle_gradients_against_differences(layout, weights):
    r = np.random.default_rng(1)
    x, dy, w = r.standard_normal((3, 2, 16)), r.standard_normal((3, 2, 16)), r.standard_normal(16) if weights else None
    turn = (np.array([[0, 5, -3], [2, 2, 9]]), np.array([1.0, 0.3, 0.2, 0.7, 0.01]), layout, (2, 3), 1.3)
    loss = lambda x, w: float((oracle.forward(x, w, 1e-3, *turn)[0] * dy).sum())  # noqa: E731
    dx, dw, _, _ = oracle.backward(x, dy, w, 1e-3, *turn)
    h = 1e-5
    for at in np.ndindex(*x.shape):
        d = np.zeros_like(x)
        d[at] = h
        assert (loss(x + d, w) - loss(x - d, w)) / (2 * h) == pytest.approx(dx[at], abs=1e-8)
    if weights:
        for j in range(16):
            d = np.zeros(16)
            d[j] = h
            assert (loss(x, w + d) - loss(x, w - d)) / (2 * h) == pytest.approx(dw[j], abs=1e-8)


def test_oracle_turn_back_is_the_transpose():
    r = np.random.default_rng(2)
    x, y = r.standard_normal((2, 4, 3, 64))
    turn = (np.arange(4)[None] * 1000, np.linspace(0.1, 2.0, 20), "half", (20,), 0.5)
    a, b = oracle.turned(x, 0 * x, *turn)[0], oracle.turned(y, 0 * y, *turn, sign=-1.0)[0]
    assert (a * y).sum() == pytest.approx((x * b).sum())


def call(which, turn=None, **kw):
    p = dict(q=A, k=A + 64 * MB, qs=768, ks=256, tokens=9, heads=6, kv_heads=2, d=128, q_out=A + 192 * MB, k_out=A + 256 * MB,
             gq=A + 320 * MB, gk=A + 384 * MB, gqs=768, gks=256, dwq=A + 448 * MB, dwk=A + 449 * MB, ws=A + 512 * MB, ws_bytes=MB)
    p.update(kw)
    t = dict(positions=A + 128 * MB, freqs=np.ones(32), sections=(32,), n=None, layout=0, mscale=1.0, eps=1e-6, wq=A + 600 * MB,
             wk=A + 601 * MB, f32=0)
    t.update(turn or {})
    sec = None if t["sections"] is None else np.ascontiguousarray(t["sections"], dtype=np.int32)
    f = None if t["freqs"] is None else np.ascontiguousarray(t["freqs"], dtype=np.float64)
    s = _lib.Turn(t["positions"], None if f is None else f.ctypes.data, None if sec is None else sec.ctypes.data,
                  t["n"] if t["n"] is not None else len(sec), t["layout"], t["mscale"], t["eps"], t["wq"], t["wk"], t["f32"])
    ref = None if turn == "none" else ctypes.byref(s)
    L, need = _lib.lib(), ctypes.c_uint64(7)
    if which == "fwd":
        st = L.t2v_norm_rotary(p["q"], p["k"], p["qs"], p["ks"], p["tokens"], p["heads"], p["kv_heads"], p["d"], ref, p["q_out"],
                               p["k_out"], None)
    else:
        st = L.t2v_norm_rotary_bwd(p["q"], p["k"], p["qs"], p["ks"], p["gq"], p["gk"], p["gqs"], p["gks"], p["tokens"], p["heads"],
                                   p["kv_heads"], p["d"], ref, p["q_out"], p["k_out"], p["dwq"], p["dwk"], p["ws"], p["ws_bytes"],
                                   ctypes.byref(need), None)
    return st, _lib.t2v_last_error(L), need.value


@pytest.mark.parametrize("which", ["fwd", "bwd"])
@pytest.mark.parametrize("turn,kw,status,msg", [
    ({}, {"d": 96}, UNS, "head_dim"), ({}, {"tokens": -1}, INV, "tokens"), ({}, {"heads": 0, "kv_heads": 0}, INV, "heads"),
    ({}, {"heads": -1}, INV, "heads"), ({}, {"heads": 1 << 16}, INV, "too large"), ({"freqs": None}, {}, INV, "NULL"),
    ({"sections": (8, 8, 8, 8)}, {}, INV, "sections"), ({"sections": (40, -8)}, {}, INV, "sections"), ({"n": -1}, {}, INV, "sections"),
    ({"layout": 2}, {}, INV, "layout"), ({"mscale": math.inf}, {}, INV, "mscale"), ({"freqs": [math.nan] * 32}, {}, INV, "freqs"),
    ({"eps": math.nan}, {}, INV, "eps"), ({"eps": math.inf}, {}, INV, "eps"), ({"eps": -1.0}, {}, INV, "q_weight"),
    ({}, {"qs": 760}, INV, "q_stride"), ({}, {"ks": 258}, INV, "k_stride"), ({}, {"q": 0}, INV, "q is NULL"),
    ({}, {"k_out": A + 192 * MB + 16}, INV, "overlaps"), ({"positions": 0}, {}, INV, "positions"),
    ({"positions": A + 192 * MB + 64}, {}, INV, "positions"), ({"positions": A + 3}, {}, INV, "aligned"), ({}, {"q": A + 8}, INV, "aligned"),
    ({"wq": A + 192 * MB}, {}, INV, "overlaps"), ({"wk": A + 600 * MB + 8}, {}, INV, "aligned"),
])
def test_refusals(which, turn, kw, status, msg):
    st, err, need = call(which, turn, **kw)
    assert st == status and msg in err, (st, err)
    assert which == "fwd" or need == 0


@pytest.mark.parametrize("turn,kw,status,msg", [
    ({"eps": -1.0, "wq": 0, "wk": 0}, {}, INV, "needs a norm"), ({"wq": 0}, {}, INV, "dq_weight"), ({}, {"gqs": 0}, INV, "dq_out_stride"),
    ({}, {"gk": 0}, INV, "dk_out is NULL"), ({}, {"dwq": A + 449 * MB + 16}, INV, "overlaps"), ({}, {"q_out": A + 320 * MB}, INV, "overlaps"),
    ({}, {"ws_bytes": 64}, WS, "workspace"), ({}, {"ws": A, "ws_bytes": MB}, INV, "overlaps"), ({}, {"ws": 0, "ws_bytes": 0}, WS, "needs"),
])
def test_backward_refusals(turn, kw, status, msg):
    st, err, need = call("bwd", turn, **kw)
    assert st == status and msg in err and (need > 0) == (status == WS), (st, err, need)


def test_empty_calls_and_missing_struct():
    none = dict(tokens=0, q=None, k=None, q_out=None, k_out=None, gq=None, gk=None)
    assert call("fwd", {"positions": 0}, **none)[0] == _lib.T2V_OK
    assert call("bwd", {"positions": 0}, dwq=None, dwk=None, **none)[0] == _lib.T2V_OK
    L = _lib.lib()
    assert L.t2v_norm_rotary(A, A + MB, 768, 256, 9, 6, 2, 128, None, A + 2 * MB, A + 3 * MB, None) == INV


def _t(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


@pytest.mark.parametrize("kw,msg", [
    ({"q": None, "k": None}, "both None"), ({"layout": "neox"}, "layout"), ({"positions": _t(8, dtype=torch.int32)}, "positions has shape"),
    ({"sections": (3, 4)}, "sum to"), ({"freqs": None}, "without freqs"), ({"freqs": None, "positions": None, "q": _t(9, 384)}, "head_dim"),
    ({"k": _t(8, 2, 64)}, "k has shape"), ({"q_weight": _t(63)}, "q_weight"), ({"q_weight": _t(64, dtype=torch.float16)}, "q_weight"),
    ({"q_weight": _t(64), "k_weight": _t(64, dtype=torch.float32)}, "same dtype"), ({"q_weight": _t(64), "eps": None}, "without a norm"),
    ({"eps": -1.0}, "eps"), ({"eps": math.nan}, "eps"), ({"k": None, "k_weight": _t(64)}, "without k"), ({}, "CUDA"),
])
def test_binding_refusals(kw, msg):
    a = dict(q=_t(9, 6, 64), k=_t(9, 2, 64), positions=_t(9, dtype=torch.int32), freqs=np.ones(8), layout="half", sections=None,
             q_weight=None, k_weight=None, eps=1e-6)
    a.update(kw)
    with pytest.raises(ValueError, match=msg):
        t2v.norm_rotary_apply(a["q"], a["k"], a["positions"], a["freqs"], a["q_weight"], a["k_weight"], a["eps"], a["layout"],
                              a["sections"])


def test_autograd_refusals():
    with pytest.raises(ValueError, match="needs a norm"):
        t2v.norm_rotary(_t(9, 6, 64), None, _t(9, dtype=torch.int32), np.ones(8), eps=None)
    with pytest.raises(ValueError, match="needs a norm"):
        t2v.norm_rotary_bwd(_t(9, 6, 64), None, _t(9, 6, 64), None, _t(9, dtype=torch.int32), np.ones(8), eps=None)
    with pytest.raises(ValueError, match="both be given"):
        t2v.norm_rotary_bwd(_t(9, 6, 64), None, None, None, _t(9, dtype=torch.int32), np.ones(8))


# ------------------------------------------------------------------------ what autograd passes on


def leaves():
    w = torch.zeros(50, 8, 64, dtype=torch.bfloat16).requires_grad_(True)
    return w, w[:, :6], w[:, 6:], *(torch.ones(64, dtype=torch.bfloat16).requires_grad_(True) for _ in range(2))


def turned(q, k, wq, wk):
    return t2v.norm_rotary(q, k, torch.zeros(50, dtype=torch.int32), np.ones(32), wq, wk)


@pytest.mark.parametrize("hooks", HOOKS, ids=["none", "pack", "unpack"])
def test_backward_describes_the_tensors_that_it_passes(calls, hooks):
    """Saved-tensor hooks may give dense copies of slices; gradients may be spread out or start anywhere."""
    w, q, k, wq, wk = leaves()
    seen = {x.data_ptr(): x for x in (q, k)}

    def unpacked(x):
        y = hooks[1](x)
        seen[y.data_ptr()] = y
        return y

    if hooks is None:
        a, b = turned(q, k, wq, wk)
    else:
        with torch.autograd.graph.saved_tensors_hooks(hooks[0], unpacked):
            a, b = turned(q, k, wq, wk)
    da = torch.zeros(1, dtype=torch.bfloat16).expand(a.shape)
    db = torch.zeros(b.numel() + 1, dtype=torch.bfloat16)[1:].view(b.shape)
    torch.autograd.grad((a, b), (w, wq, wk), (da, db))
    args = [x for n, x in calls.made if n == "t2v_norm_rotary_bwd"][-1]
    for p, step in zip(args[0:2], args[2:4]):
        assert step == seen[p].stride(0) and p % 16 == 0
    assert all(p % 16 == 0 and p for p in args[4:6]) and args[6:8] == (6 * 64, 2 * 64)


@pytest.mark.parametrize("eager,refused", [(0, True), (7, False), (None, False)], ids=["default stream", "side stream", "no eager graph"])
def test_captured_backward_beside_an_eager_graph(calls, monkeypatch, eager, refused):
    w, q, k, wq, wk = leaves()
    current = [eager or 0]
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: current[0], raising=False)
    alive = turned(q, k, wq, wk) if eager is not None else None
    current[0] = 9
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    out = turned(q, k, wq, wk)
    g = tuple(torch.zeros_like(x) for x in out)
    if refused:
        with pytest.raises(RuntimeError, match="default stream"):
            torch.autograd.grad(out, (wq, wk), g)
        del alive, out
        out = turned(q, k, wq, wk)
    torch.autograd.grad(out, (wq, wk), g)
