"""The forward form for at most 32 packed rows (single tokens, short chunks) with what the other forms are tested with: scales of
any sign, masked infinities and NaN, scores of -inf, waves that see no key, cut loops; and caches with room behind each sequence."""
import ctypes

import numpy as np
import pytest
import torch

import oracle
from paper_2607_01701_amd import _lib, causal_attn_bwd, causal_attn_fwd

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
    return mk(lq, H), mk(lk, Hk), mk(lk, Hk)


def forward(q, k, v, lq, lk, scale):
    nan = lambda *s, dtype: torch.full(s, float("nan"), dtype=dtype, device="cuda")  # noqa: E731
    out, lse = causal_attn_fwd(q, k, v, cu(lq), scale, nan(*q.shape, dtype=torch.bfloat16),
                               nan(q.shape[1], q.shape[0], dtype=torch.float32), cu_seqlens_k=cu(lk))
    torch.cuda.synchronize()
    return out, lse


def is_cut(q, k, lq, lk):
    """Whether the call cuts its loops: it then needs a workspace."""
    need, (T, H, D), Hk, a, b = ctypes.c_uint64(0), q.shape, k.shape[1], cu(lq), cu(lk)
    out, lse = torch.empty_like(q), torch.empty((H, T), device="cuda")
    _lib.lib().t2v_causal_fwd(q.data_ptr(), k.data_ptr(), k.data_ptr(), H * D, Hk * D, Hk * D, _lib._offsets_ptr(a),
                              _lib._offsets_ptr(b), len(lq), H, Hk, D, 0.1, out.data_ptr(), lse.data_ptr(), None, 0,
                              ctypes.byref(need), None)
    torch.cuda.synchronize()
    return need.value > 0


def check(out, lse, ref):
    for name, got in (("out", out), ("lse", lse)):
        g, r, b = got.double().cpu().numpy(), ref[name], ref["bounds"][name]
        assert np.array_equal(np.isneginf(g), np.isneginf(r)), name
        fin = np.isfinite(r)
        worst = float((np.abs(np.where(fin, g - np.where(fin, r, 0.0), 0.0)) / (b + 1e-30)).max())
        log(f"{name}: {worst:.3f} of the bound")
        assert worst <= 1.0, name


# One whole, one cut; waves without keys (few of them), and queries without any.
SHAPES = [([4], [300], False), ([4, 1], [9001, 77], True), ([3, 5, 2, 1], [5, 33, 1, 0], False)]


@pytest.mark.parametrize("scale", [0.0, -0.3, 1.0])
@pytest.mark.parametrize("lq,lk,cut", SHAPES)
@pytest.mark.parametrize("H,Hk,D", [(4, 2, 64), (4, 2, 128)])
def test_scales(lq, lk, cut, H, Hk, D, scale):
    log(f"case few rows {lq} over {lk} {H}/{Hk}x{D} scale {scale}")
    q, k, v = pack(lq, lk, H, Hk, D, 1)
    assert is_cut(q, k, lq, lk) == cut
    out, lse = forward(q, k, v, lq, lk, scale)
    check(out, lse, oracle.causal_attention(*(x.float().cpu().numpy() for x in (q, k, v)), None, cu(lq), cu(lk), scale))


@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("lk", [300, 9001, 6])
@pytest.mark.parametrize("H,Hk,D", [(4, 2, 64), (4, 2, 128)])
def test_what_a_query_does_not_see_does_not_reach_it(H, Hk, D, lk, what):
    log(f"case few rows masked {what} over {lk} {H}/{Hk}x{D}")
    lq, at = [4], lk - 2  # queries 2 and 3 see it
    q, k, v = pack(lq, [lk], H, Hk, D, 2)
    assert is_cut(q, k, lq, [lk]) == (lk == 9001)
    clean, clean_lse = forward(q, k, v, lq, [lk], 0.1)
    k2, v2 = k.clone(), v.clone()
    k2[at, 0], v2[at, 1, 3] = what, what
    out, lse = forward(q, k2, v2, lq, [lk], 0.1)
    assert torch.equal(out[:2], clean[:2]) and torch.equal(lse[:, :2], clean_lse[:, :2])
    assert not torch.isfinite(out[2:, 2:, 3]).any() and not torch.isfinite(out[2:, :2]).any()
    other = [d for d in range(D) if d != 3]
    assert torch.equal(out[:, 2:][..., other], clean[:, 2:][..., other]) and torch.equal(lse[2:], clean_lse[2:])
    v3 = v.clone()
    v3[0, 0, 5] = what  # every query sees it
    out, lse = forward(q, k, v3, lq, [lk], 0.1)
    assert not torch.isfinite(out[:, :2, 5]).any() and torch.equal(out[:, 2:], clean[:, 2:]) and torch.equal(lse, clean_lse)


@pytest.mark.parametrize("lk", [300, 9001])
@pytest.mark.parametrize("D", [64, 128])
def test_scores_of_minus_infinity_weigh_nothing(D, lk):
    log(f"case few rows, scores of -inf over {lk} x{D}")
    lq, H, Hk = [3], 4, 2
    q, k, v = pack(lq, [lk], H, Hk, D, 3)
    q[..., 0] = q[..., 0].abs() + 0.5
    dead = torch.rand(lk, generator=torch.Generator().manual_seed(4)) < 0.5
    dead[:64] = True  # whole steps of a wave, and the first key of the first query
    dead[100] = False
    k[dead.cuda()] = 0.0
    k[dead.cuda(), :, 0] = -float("inf")
    out, lse = forward(q, k, v, lq, [lk], 0.1)
    with np.errstate(invalid="ignore"):
        ref = oracle.causal_attention(*(x.float().cpu().numpy() for x in (q, k, v)), None, cu(lq), cu([lk]), 0.1)
    finite = k.float().cpu().numpy()
    finite[dead.numpy()] = 0.0  # the bound of lse: that of the other keys
    ref["bounds"]["lse"] = oracle.causal_attention(q.float().cpu().numpy(), finite, finite, None, cu(lq), cu([lk]), 0.1)["bounds"]["lse"]
    check(out, lse, ref)


@pytest.mark.parametrize("lq,lk,H,Hk,D", [([1] * 4, [700, 5, 3000, 64], 8, 2, 128), ([1, 1], [1280, 2], 30, 10, 64),
                                          ([40, 3, 1], [900, 3, 77], 6, 2, 128)])
def test_caches_with_room_behind_each_sequence(lq, lk, H, Hk, D):
    """A sequence without queries in the place of each gap: the results are those of caches packed without gaps, bitwise, whatever
    the gaps hold; and the gaps' gradients are zero."""
    log(f"case caches with room {lq} over {lk} {H}/{Hk}x{D}")
    room = max(lk) + 13
    q, k, v = pack(lq, lk, H, Hk, D, 5)
    want, want_lse = forward(q, k, v, lq, lk, 0.1)
    kc, vc = (torch.full((len(lk), room, Hk, D), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    at = cu(lk)
    for i, n in enumerate(lk):
        kc[i, :n], vc[i, :n] = k[at[i]:at[i + 1]], v[at[i]:at[i + 1]]
    gap_q, gap_k = [x for n in lq for x in (n, 0)], [x for n in lk for x in (n, room - n)]
    kc, vc = kc.view(-1, Hk, D), vc.view(-1, Hk, D)
    out, lse = forward(q, kc, vc, gap_q, gap_k, 0.1)
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    g = pack(lq, lk, H, Hk, D, 6)[0]
    grads = causal_attn_bwd(q, k, v, want, want_lse, g, cu(lq), 0.1, cu_seqlens_k=cu(lk))
    dq, dk, dv = causal_attn_bwd(q, kc, vc, out, lse, g, cu(gap_q), 0.1, cu_seqlens_k=cu(gap_k))
    torch.cuda.synchronize()
    b = oracle.causal_attention(*(x.float().cpu().numpy() for x in (q, k, v, g)), cu(lq), cu(lk), 0.1)["bounds"]
    assert ((dq.double() - grads[0].double()).abs().cpu().numpy() <= 2 * b["dq"] + 1e-30).all()
    for got, whole, name in ((dk, grads[1], "dk"), (dv, grads[2], "dv")):
        got = got.view(len(lk), room, Hk, D)
        assert all((got[i, n:] == 0).all() for i, n in enumerate(lk)), name
        kept = torch.cat([got[i, :n] for i, n in enumerate(lk)])  # the cuts may differ, the results only by rounding
        assert ((kept.double() - whole.double()).abs().cpu().numpy() <= 2 * b[name] + 1e-30).all(), name
