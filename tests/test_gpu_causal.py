"""Causal attention with grouped heads on the GPU, element by element against the float64 oracle and within
its derived bounds: head layouts, lengths around the tiles, rows without keys, chunks and single tokens over
long caches (cut loops), slices of a fused projection, scales, masked infinities and NaN."""
import numpy as np
import pytest
import torch

import oracle
from paper_2607_01701_amd import (T2VError, _lib, causal_attn_bwd, causal_attn_fwd, use_checked_library,
                                  varlen_causal_attention)

from gpu_util import log

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def cu(lengths):
    return np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)


def pack(lq, lk, H, Hk, D, seed):
    g = torch.Generator().manual_seed(seed)
    mk = lambda t, h: torch.randn((sum(t), h, D), generator=g).bfloat16().cuda()  # noqa: E731
    return mk(lq, H), mk(lk, Hk), mk(lk, Hk), mk(lq, H)


def run(q, k, v, dout, cq, ck, scale):
    """Forward and backward into poisoned outputs."""
    (Tq, H, D), (Tk, Hk, _) = q.shape, k.shape
    nan = lambda *s, dtype=torch.bfloat16: torch.full(s, float("nan"), dtype=dtype, device="cuda")  # noqa: E731
    out, lse = causal_attn_fwd(q, k, v, cq, scale, nan(Tq, H, D), nan(H, Tq, dtype=torch.float32), cu_seqlens_k=ck)
    dq, dk, dv = causal_attn_bwd(q, k, v, out, lse, dout, cq, scale, nan(Tq, H, D), nan(Tk, Hk, D), nan(Tk, Hk, D),
                                 nan(2, H, Tq, dtype=torch.float32), cu_seqlens_k=ck)
    torch.cuda.synchronize()
    return {"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv}


def check(got, ref, names=("out", "lse", "dq", "dk", "dv")):
    worst = {}
    for n in names:
        g, r, b = got[n].double().cpu().numpy(), ref[n], ref["bounds"][n]
        assert g.shape == r.shape
        if g.size == 0:
            continue
        fin = np.isfinite(r)
        assert np.array_equal(np.isneginf(g), np.isneginf(r)), n
        e = np.abs(np.where(fin, g - np.where(fin, r, 0.0), 0.0))
        assert not np.isnan(e).any(), f"{n}: NaN"
        worst[n] = float((e / (b + 1e-30)).max())
    log(f"errors as shares of their bounds: { {n: round(x, 3) for n, x in worst.items()} }")
    for n, x in worst.items():
        assert x <= 1.0, f"{n} is {x:.2f} times its bound off"


EDGES = [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300]
SAME = [(EDGES, 2, 2, 128), (EDGES, 4, 1, 64), (EDGES, 6, 2, 128), ([0, 700, 0, 1, 513], 3, 1, 64),
        ([1000, 257], 5, 5, 128), ([640, 255], 16, 1, 64), ([333], 7, 1, 128), ([1500], 2, 1, 64)]


@pytest.fixture(params=["", "wide", "narrow"])
def tiles(request, monkeypatch):
    """The forms that the library would choose, and each of them forced."""
    for name in ("T2V_QTILE", "T2V_KVTILE"):
        monkeypatch.setenv(name, request.param)
    return request.param or "chosen"


@pytest.mark.parametrize("lengths,H,Hk,D", SAME)
def test_prompts(lengths, H, Hk, D, tiles):
    log(f"case prompts {lengths} {H}/{Hk}x{D} {tiles} tiles")
    p = pack(lengths, lengths, H, Hk, D, 1)
    c = cu(lengths)
    got = run(*p, c, None, D ** -0.5)
    check(got, oracle.causal_attention(*(x.float().cpu().numpy() for x in p), c, c, D ** -0.5))


CHUNKS = [([1, 1, 1], [1, 77, 2049], 8, 2, 128), ([1] * 5, [64, 65, 3000, 1, 128], 40, 8, 128),
          ([3, 1, 16], [700, 5000, 16], 30, 10, 64), ([100, 33, 257], [1000, 33, 4100], 6, 3, 128),
          ([5, 64, 2, 0, 7], [3, 10, 0, 9, 0], 4, 2, 64), ([200], [100], 2, 1, 128), ([2], [9001], 2, 2, 64)]


@pytest.mark.parametrize("lq,lk,H,Hk,D", CHUNKS)
def test_chunks_over_a_cache(lq, lk, H, Hk, D, tiles):
    log(f"case chunks {lq} over {lk} {H}/{Hk}x{D} {tiles} tiles")
    p = pack(lq, lk, H, Hk, D, 2)
    got = run(*p, cu(lq), cu(lk), D ** -0.5)
    check(got, oracle.causal_attention(*(x.float().cpu().numpy() for x in p), cu(lq), cu(lk), D ** -0.5))


@pytest.mark.parametrize("scale", [0.0, -0.3, 1.0])
def test_scales(scale):
    log(f"case scale {scale}")
    p = pack([130, 40], [200, 40], 4, 2, 64, 3)
    got = run(*p, cu([130, 40]), cu([200, 40]), scale)
    check(got, oracle.causal_attention(*(x.float().cpu().numpy() for x in p), cu([130, 40]), cu([200, 40]), scale))


def test_slices_of_a_fused_projection():
    log("case fused slices")
    H, Hk, D, n = 6, 2, 128, [300, 77]
    qkv = torch.randn(377, H + 2 * Hk + 1, D, generator=torch.Generator().manual_seed(4)).bfloat16().cuda()
    q, k, v = qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:H + 2 * Hk]
    g = torch.randn(377, H, D, generator=torch.Generator().manual_seed(5)).bfloat16().cuda()
    a, b = run(q, k, v, g, cu(n), None, 0.1), run(q.contiguous(), k.contiguous(), v.contiguous(), g, cu(n), None, 0.1)
    for name in a:
        assert torch.equal(a[name], b[name]), name


@pytest.mark.parametrize("what", [float("nan"), float("inf")])
@pytest.mark.parametrize("D", [64, 128])
def test_what_a_query_does_not_see_does_not_reach_it(what, D, tiles):
    """Later keys and values of infinities and NaN leave earlier rows' results as they are, and a query's own
    reach only the keys that it sees."""
    log(f"case masked {what} D={D} {tiles} tiles")
    n, at, H, Hk = 350, 70, 4, 2
    q, k, v, g = pack([n], [n], H, Hk, D, 6)
    clean = run(q, k, v, g, cu([n]), None, 0.1)
    k2, v2 = k.clone(), v.clone()
    k2[at, 0], v2[at, 1, 3] = what, what
    got = run(q, k2, v2, g, cu([n]), None, 0.1)
    for name in ("out", "dq"):
        assert torch.equal(got[name][:at], clean[name][:at]), name
    assert torch.equal(got["lse"][:, :at], clean["lse"][:, :at])
    assert not torch.isfinite(got["out"][at:, 2:, 3]).any()
    assert torch.isfinite(got["out"][at:, 2:, 4]).all()
    q2, g2 = q.clone(), g.clone()
    g2[at, 1], q2[at, 2] = what, what
    got = run(q2, k, v, g2, cu([n]), None, 0.1)
    for name in ("dk", "dv"):
        assert torch.equal(got[name][at + 1:], clean[name][at + 1:]), name
        assert not torch.isfinite(got[name][:at + 1]).any(), name
    # the last query, whose step is partial, sees every key
    g3 = g.clone()
    g3[n - 1, 0, 5] = what
    got = run(q, k, v, g3, cu([n]), None, 0.1)
    assert not torch.isfinite(got["dv"][:, 0, 5]).any() and torch.equal(got["dv"][:, 1], clean["dv"][:, 1])
    assert torch.equal(got["dv"][:, 0, 6], clean["dv"][:, 0, 6])


def test_autograd_equals_the_calls_and_repeats_bitwise():
    log("case autograd")
    p = pack([400, 31], [900, 31], 6, 2, 128, 7)
    a = run(*p, cu([400, 31]), cu([900, 31]), 0.09)
    q, k, v = (x.clone().requires_grad_(True) for x in p[:3])
    out, lse = varlen_causal_attention(q, k, v, cu([400, 31]), 0.09, cu_seqlens_k=cu([900, 31]))
    out.backward(p[3])
    for x, name in ((out, "out"), (lse, "lse"), (q.grad, "dq"), (k.grad, "dk"), (v.grad, "dv")):
        assert torch.equal(x, a[name]), name


def test_checked_library_gives_the_same(tiles):
    for lq, lk, H, Hk, D in [*CHUNKS, *((n, n, *r) for n, *r in SAME)]:
        log(f"case checked {lq} {lk} {H}/{Hk}x{D}")
        p = pack(lq, lk, H, Hk, D, 8)
        a = run(*p, cu(lq), cu(lk), 0.1)
        with use_checked_library():
            b = run(*p, cu(lq), cu(lk), 0.1)
        for name in a:
            assert torch.equal(a[name], b[name]), name


def test_empty_calls():
    z = torch.zeros((0, 4, 64), dtype=torch.bfloat16, device="cuda")
    k = torch.ones((5, 2, 64), dtype=torch.bfloat16, device="cuda")
    got = run(z, k, k, z, cu([0]), cu([5]), 0.1)
    assert (got["dk"] == 0).all() and (got["dv"] == 0).all() and got["out"].numel() == 0
    q = torch.ones((5, 4, 64), dtype=torch.bfloat16, device="cuda")
    got = run(q, z[:, :2], z[:, :2], q, cu([5]), cu([0]), 0.1)
    assert (got["out"] == 0).all() and (got["dq"] == 0).all() and torch.isneginf(got["lse"]).all()
    run(z, z[:, :2], z[:, :2], z, cu([0]), None, 0.1)
    assert _lib.T2V_OK == 0


def test_checked_library_reports_rows_out_of_bounds(tiles, monkeypatch):
    """With a row taken off every bound, correct kernels report their sequences' last rows: each kernel checks its copies."""
    monkeypatch.setenv("T2V_CHECK_CANARY", "1")
    for lq, lk, H, Hk, D in (([70], [70], 4, 2, 128), ([300], [300], 2, 2, 64), ([1], [90], 4, 2, 64)):
        log(f"case canary {lq} {lk} {tiles} tiles")
        q, k, v, g = pack(lq, lk, H, Hk, D, 9)
        out, lse = causal_attn_fwd(q, k, v, cu(lq), 0.1, cu_seqlens_k=cu(lk))
        with use_checked_library():
            with pytest.raises(T2VError, match="causal forward kernel"):
                causal_attn_fwd(q, k, v, cu(lq), 0.1, cu_seqlens_k=cu(lk))
            with pytest.raises(T2VError, match="causal dK/dV kernel"):
                causal_attn_bwd(q, k, v, out, lse, g, cu(lq), 0.1, cu_seqlens_k=cu(lk))
    monkeypatch.delenv("T2V_CHECK_CANARY")
    with use_checked_library():
        causal_attn_fwd(q, k, v, cu(lq), 0.1, cu_seqlens_k=cu(lk))
