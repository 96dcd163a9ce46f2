"""The causal attention and rotary calls on the CPU: refusals before anything is launched, by the C ABI (fake
addresses, never dereferenced) and by the binding; empty calls; rotary frequencies."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2607_01701_amd as t2v
from paper_2607_01701_amd import _lib

A, MB = 0x100000, 1 << 20
INV, UNS = _lib.T2V_ERR_INVALID_ARG, _lib.T2V_ERR_UNSUPPORTED


def _i32(x):
    return np.ascontiguousarray(x, dtype=np.int32)


def _ptr(x):
    return None if x is None else x.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))


def call(which, cu=(0, 5, 9), cu_k=(0, 7, 20), **kw):
    p = dict(q=A, k=A + 64 * MB, v=A + 128 * MB, out=A + 192 * MB, lse=A + 256 * MB, dout=A + 320 * MB, dq=A + 384 * MB,
             dk=A + 448 * MB, dv=A + 512 * MB, delta=A + 576 * MB, heads=6, kv_heads=2, head_dim=128, scale=0.1, qs=None,
             ks=None, vs=None, ws=None, ws_bytes=0, nseq=None)
    p.update(kw)
    h, hk, d = p["heads"], p["kv_heads"], p["head_dim"]
    strides = [s if s is not None else n * d for s, n in ((p["qs"], h), (p["ks"], hk), (p["vs"], hk))]
    cq = None if cu is None else _i32(cu)
    ck = None if cu_k is None else _i32(cu_k)
    n = p["nseq"] if p["nseq"] is not None else (len(cq) - 1 if cq is not None else 1)
    L, need = _lib.lib(), ctypes.c_uint64(7)
    tail = (p["ws"], p["ws_bytes"], ctypes.byref(need), None)
    if which == "fwd":
        st = L.t2v_causal_fwd(p["q"], p["k"], p["v"], *strides, _ptr(cq), _ptr(ck), n, h, hk, d, p["scale"], p["out"],
                              p["lse"], *tail)
    else:
        st = L.t2v_causal_bwd(p["q"], p["k"], p["v"], *strides, p["out"], p["lse"], _ptr(cq), _ptr(ck), n, h, hk, d,
                              p["scale"], p["dout"], p["dq"], p["dk"], p["dv"], p["delta"], *tail)
    return st, _lib.t2v_last_error(L), need.value


BOTH = [
    ({"cu": (1, 5)}, INV, "cu_seqlens[0]"), ({"cu": (0, 5, 3)}, INV, "non-decreasing"),
    ({"cu_k": (0, 5, 3)}, INV, "cu_seqlens_k"), ({"cu": None}, INV, "NULL"), ({"cu_k": None}, INV, "NULL"),
    ({"nseq": -1}, INV, "nseq"), ({"heads": 0}, INV, "multiple"), ({"kv_heads": 0}, INV, "multiple"),
    ({"heads": 7}, INV, "multiple"), ({"heads": 2, "kv_heads": 4}, INV, "multiple"), ({"head_dim": 96}, UNS, "head_dim"),
    ({"scale": float("nan")}, INV, "scale"), ({"qs": 6 * 128 - 8}, INV, "q_stride"), ({"ks": 260}, INV, "k_stride"),
    ({"vs": (1 << 22) + 8}, INV, "v_stride"), ({"vs": 0}, INV, "v_stride"), ({"q": 0}, INV, "q is NULL"),
    ({"k": A + 64 * MB + 8}, INV, "aligned"), ({"lse": 0}, INV, "lse is NULL"),
    ({"heads": 1 << 16, "kv_heads": 1, "cu": (0, 40000, 80000), "cu_k": (0, 1, 2)}, INV, ""),
    ({"ws": A + 16, "ws_bytes": 4096}, INV, "overlaps"), ({"ws": A + 640 * MB + 4, "ws_bytes": 64}, INV, "aligned"),
    ({"ws": None, "ws_bytes": 64}, INV, "ws is NULL"),
]


@pytest.mark.parametrize("which", ["fwd", "bwd"])
@pytest.mark.parametrize("kw,status,msg", BOTH)
def test_refusals(which, kw, status, msg):
    st, err, need = call(which, **kw)
    assert st == status and msg in err and need == 0, (st, err, need)


@pytest.mark.parametrize("which,kw,msg", [
    ("fwd", {"out": A + 64}, "overlaps"), ("fwd", {"lse": A + 192 * MB}, "overlaps"),
    ("fwd", {"out": A + (4 * 800 + 6 * 128) * 2, "qs": 840}, "overlaps"),  # in the last token's rows
    ("bwd", {"dq": A + 448 * MB}, "overlaps"), ("bwd", {"dv": A}, "overlaps"), ("bwd", {"delta": A + 320 * MB}, "overlaps"),
    ("bwd", {"dout": 0}, "dout is NULL"), ("bwd", {"delta": 0}, "delta_ws is NULL"), ("bwd", {"dk": A + 448 * MB + 2}, "aligned"),
])
def test_pointers(which, kw, msg):
    st, err, _ = call(which, **kw)
    assert st == INV and msg in err, (st, err)


def test_too_many_rows_of_a_group():
    # 2^31 packed rows of one sequence: refused although each tensor's size would pass.
    st, err, _ = call("fwd", cu=(0, 1 << 26), cu_k=(0, 1), heads=64, kv_heads=1, head_dim=64)
    assert st == INV and "too many queries" in err, (st, err)


def test_empty_calls_need_no_pointers():
    none = dict(q=None, k=None, v=None, out=None, lse=None, dout=None, dq=None, dk=None, dv=None, delta=None)
    for which in ("fwd", "bwd"):
        assert call(which, cu=(0, 0, 0), cu_k=(0, 0, 0), **none)[0] == _lib.T2V_OK
        assert call(which, cu=(0,), cu_k=(0,), **none)[0] == _lib.T2V_OK
    assert call("fwd", cu=(0, 0), cu_k=(0, 9), **none)[0] == _lib.T2V_OK  # keys without queries: no output
    st, err, _ = call("bwd", cu=(0, 0), cu_k=(0, 9), **none)  # but their gradients are written
    assert st == INV and "NULL" in err


def _t(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


@pytest.mark.parametrize("change,msg", [
    ({"k": _t(20, 2, 64)}, "k has shape"), ({"v": _t(19, 2, 128)}, "v has shape"),
    ({"q": _t(9, 6, 128, dtype=torch.float16)}, "dtype"), ({"q": _t(9, 6 * 128)}, "head_dim"),
    ({"q": _t(6, 9, 128).transpose(0, 1)}, "contiguously"), ({"k": _t(20, 2, 256)[..., ::2]}, "contiguously"),
    ({"q": _t(1, 6, 128).expand(9, 6, 128)}, "contiguously"),
    ({"cu": [0, 5, 8]}, "does not match"), ({"cu_k": [0, 7, 21]}, "does not match"), ({"cu_k": [0, 20]}, "entries"),
    ({"cu_k": None}, "does not match"), ({}, "must be a CUDA tensor"),
])
def test_binding_refusals(change, msg):
    a = dict(q=_t(9, 6, 128), k=_t(20, 2, 128), v=_t(20, 2, 128), cu=[0, 5, 9], cu_k=[0, 7, 20])
    a.update(change)
    with pytest.raises(ValueError, match=msg):
        t2v.causal_attn_fwd(a["q"], a["k"], a["v"], a["cu"], 0.1, cu_seqlens_k=a["cu_k"])
    if not msg.startswith("must be"):  # the backward call checks the same first
        with pytest.raises(ValueError, match=msg):
            t2v.causal_attn_bwd(a["q"], a["k"], a["v"], None, None, None, a["cu"], 0.1, cu_seqlens_k=a["cu_k"])


def rot(**kw):
    p = dict(q=A, k=A + 64 * MB, qs=768, ks=256, pos=A + 128 * MB, tokens=9, heads=6, kv_heads=2, d=128, freqs=np.ones(32),
             sections=(32,), n=None, layout=0, mscale=1.0, q_out=A + 192 * MB, k_out=A + 256 * MB)
    p.update(kw)
    sec = None if p["sections"] is None else _i32(p["sections"])
    f = None if p["freqs"] is None else np.ascontiguousarray(p["freqs"], dtype=np.float64)
    L = _lib.lib()
    st = L.t2v_rotary(p["q"], p["k"], p["qs"], p["ks"], p["pos"], p["tokens"], p["heads"], p["kv_heads"], p["d"],
                      None if f is None else f.ctypes.data, _ptr(sec), p["n"] if p["n"] is not None else len(sec) if sec is
                      not None else 1, p["layout"], p["mscale"], 0, p["q_out"], p["k_out"], None)
    return st, _lib.t2v_last_error(L)


@pytest.mark.parametrize("kw,status,msg", [
    ({"d": 96}, UNS, "head_dim"), ({"tokens": -1}, INV, "tokens"), ({"heads": 0, "kv_heads": 0}, INV, "heads"),
    ({"heads": -1}, INV, "heads"), ({"heads": 1 << 16}, INV, "too large"), ({"freqs": None}, INV, "NULL"),
    ({"sections": None}, INV, "NULL"), ({"n": 0}, INV, "sections"), ({"sections": (8, 8, 8, 8)}, INV, "sections"),
    ({"sections": (40, -8)}, INV, "sections"), ({"sections": (0,)}, INV, "sections"), ({"sections": (65,), "freqs": np.ones(65)}, INV, "sections"),
    ({"layout": 2}, INV, "layout"), ({"mscale": math.inf}, INV, "mscale"), ({"freqs": [math.nan] * 32}, INV, "freqs"),
    ({"qs": 760}, INV, "q_stride"), ({"ks": 258}, INV, "k_stride"), ({"q": 0}, INV, "q is NULL"), ({"k_out": 0}, INV, "k_out is NULL"),
    ({"q_out": A + 128}, INV, "overlaps"), ({"k_out": A + 192 * MB + 16}, INV, "overlaps"), ({"pos": 0}, INV, "positions"),
    ({"pos": A + 192 * MB + 64}, INV, "positions"), ({"pos": A + 3}, INV, "aligned"), ({"q": A + 8}, INV, "aligned"),
])
def test_rotary_refusals(kw, status, msg):
    st, err = rot(**kw)
    assert st == status and msg in err, (st, err)


def test_rotary_empty_call():
    assert rot(tokens=0, q=None, k=None, pos=None, q_out=None, k_out=None)[0] == _lib.T2V_OK


@pytest.mark.parametrize("kw,msg", [
    ({"q": None, "k": None}, "both None"), ({"layout": "neox"}, "layout"), ({"positions": _t(8, dtype=torch.int32)}, "positions has shape"),
    ({"positions": _t(9, dtype=torch.int64)}, "int32"), ({"sections": (3, 4)}, "sum to"), ({"sections": (2, 2, 2, 2)}, "one to three"),
    ({"sections": (4, 4)}, "positions has shape"), ({"freqs": np.ones((2, 4))}, "1-D"), ({"k": _t(8, 2, 64)}, "k has shape"),
    ({}, "CUDA"),
])
def test_rotary_binding_refusals(kw, msg):
    a = dict(q=_t(9, 6, 64), k=_t(9, 2, 64), positions=_t(9, dtype=torch.int32), freqs=np.ones(8), layout="half", sections=None)
    a.update(kw)
    with pytest.raises(ValueError, match=msg):
        t2v.rotary_apply(a["q"], a["k"], a["positions"], a["freqs"], a["layout"], a["sections"])


def test_frequencies():
    f, m = t2v.rotary_frequencies(32, 10000.0)
    assert m == 1.0 and f.shape == (32,) and f[0] == 1.0 and f[31] == pytest.approx(10000.0 ** (-31 / 32))
    axes, _ = t2v.rotary_frequencies((16, 24, 24))
    assert axes.shape == (64,) and axes[16] == 1.0 and axes[17] == pytest.approx(10000.0 ** (-1 / 24))
    lin, _ = t2v.rotary_frequencies(32, scaling="linear", factor=4.0)
    assert np.allclose(lin, f / 4.0)
    ntk, _ = t2v.rotary_frequencies(32, scaling="ntk", factor=4.0)
    assert ntk[0] == 1.0 and ntk[31] == pytest.approx(f[31] / 4.0)
    y, m = t2v.rotary_frequencies(32, scaling="yarn", factor=4.0, trained=4096)
    turns = 4096 * f / (2 * np.pi)
    assert np.allclose(y[turns >= 32], f[turns >= 32]) and np.allclose(y[turns <= 1], f[turns <= 1] / 4.0)
    assert m == pytest.approx(0.1 * math.log(4.0) + 1.0)
    assert (np.diff(y) < 0).all()
    for bad in (dict(sections=()), dict(sections=0), dict(sections=(1, 2, 3, 4)), dict(sections=4, scaling="other"),
                dict(sections=4, theta=-1.0), dict(sections=4, factor=0.0), dict(sections=4, scaling="yarn")):
        with pytest.raises(ValueError):
            t2v.rotary_frequencies(**bad)
