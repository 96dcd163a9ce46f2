"""Causal attention and rotary positions as a program uses them: together, on other streams, captured into graphs and
replayed, from several threads, over caches beyond 32-bit offsets, and with outputs in larger buffers."""
import ctypes
import threading

import numpy as np
import pytest
import torch

import oracle
import paper_2607_01701_amd as t2v
from paper_2607_01701_amd import _lib

from gpu_util import log

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def cu(lengths):
    return np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)


def rand(*shape, seed=0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).bfloat16().cuda()


def positions(lengths, start=0):
    return torch.cat([torch.arange(start, start + n, dtype=torch.int32) for n in lengths]).cuda()


def test_rotary_then_attention_trains_and_answers():
    """A block's own use: queries, keys and values from one projection, rotary positions, causal attention; its gradients;
    then the same answer token by token over the cached keys and values."""
    log("case block")
    H, Hk, D, n = 6, 2, 128, [70, 41]
    T, c, scale = sum(n), cu(n), 0.09
    w = rand(T, H + 2 * Hk, D, seed=1).requires_grad_(True)
    g = rand(T, H, D, seed=2)
    freqs, m = t2v.rotary_frequencies(40, scaling="yarn", factor=4.0, trained=64)
    pos = positions(n, 1000)
    q, k = t2v.rotary(w[:, :H], w[:, H:H + Hk], pos, freqs, mscale=m)
    out, lse = t2v.varlen_causal_attention(q, k, w[:, H + Hk:], c, scale)
    out.backward(g)
    torch.cuda.synchronize()
    # The definition in float64, with q and k rounded where the calls round them.
    x = w.detach().double().cpu().numpy()
    angle = pos.cpu().numpy()[:, None].astype(np.float64) * freqs
    cos, sin = np.cos(angle)[:, None] * m, np.sin(angle)[:, None] * m

    def turn(y, s):
        z, a, b = y.copy(), y[..., :40], y[..., 40:80]
        z[..., :40], z[..., 40:80] = a * cos - s * b * sin, s * a * sin + b * cos
        return z

    exact = [turn(x[:, :H], 1.0), turn(x[:, H:H + Hk], 1.0)]
    for got, ref in zip((q, k), exact):
        assert np.abs(got.detach().double().cpu().numpy() - ref).max() <= 2.0 ** -8 * np.abs(ref).max() + 1e-6
    ref = oracle.causal_attention(q.detach().float().cpu().numpy(), k.detach().float().cpu().numpy(), x[:, H + Hk:],
                                  g.float().cpu().numpy(), c, c, scale)
    assert (np.abs(out.detach().double().cpu().numpy() - ref["out"]) <= ref["bounds"]["out"] + 1e-30).all()
    grad = w.grad.double().cpu().numpy()
    b = ref["bounds"]
    assert (np.abs(grad[:, H + Hk:] - ref["dv"]) <= b["dv"] + 1e-30).all()
    for got, d, bound in ((grad[:, :H], ref["dq"], b["dq"]), (grad[:, H:H + Hk], ref["dk"], b["dk"])):
        want = turn(d, -1.0)
        # Rotating back mixes two elements' errors, and rounds once more.
        mixed = bound.copy()
        mixed[..., :40] = mixed[..., 40:80] = abs(m) * (bound[..., :40] + bound[..., 40:80])
        assert (np.abs(got - want) <= mixed * 1.01 + 2.0 ** -8 * (np.abs(want) + mixed) + 1e-6).all()
    # Token by token: query i over keys 0 .. i.
    for i in (0, 1, 40):
        rows = [i, n[0] + min(i, n[1] - 1)]
        keys = torch.cat([k.detach()[:i + 1], k.detach()[n[0]:rows[1] + 1]])
        vals = torch.cat([w.detach()[:i + 1, H + Hk:], w.detach()[n[0]:rows[1] + 1, H + Hk:]]).contiguous()
        one, one_lse = t2v.causal_attn_fwd(q.detach()[rows].contiguous(), keys, vals, cu([1, 1]), scale,
                                           cu_seqlens_k=cu([i + 1, rows[1] + 1 - n[0]]))
        torch.cuda.synchronize()
        assert (np.abs(one.double().cpu().numpy() - ref["out"][rows]) <= b["out"][rows] + 1e-30).all()
        assert (np.abs(one_lse.double().cpu().numpy() - ref["lse"][:, rows]) <= b["lse"][:, rows]).all()


@pytest.mark.parametrize("D", [64, 128])
def test_tile_shapes_and_workspaces_do_not_change_results(D, monkeypatch):
    """Where no loop is cut, the shape of a tile of rows is a choice of speed alone; so is the size of the workspace that a
    call offers first."""
    log(f"case shapes D={D}")
    n, H, Hk = [700, 33, 260], 6, 2
    q, k, v, g = rand(993, H, D, seed=1), rand(993, Hk, D, seed=2), rand(993, Hk, D, seed=3), rand(993, H, D, seed=4)

    def run():
        out, lse = t2v.causal_attn_fwd(q, k, v, cu(n), 0.1)
        r = (out, lse, *t2v.causal_attn_bwd(q, k, v, out, lse, g, cu(n), 0.1))
        torch.cuda.synchronize()
        return r

    want = run()
    for offered in (1, 1 << 26):
        monkeypatch.setattr(_lib, "_WORKSPACE", offered)
        assert all(torch.equal(a, b) for a, b in zip(run(), want))
    monkeypatch.setenv("T2V_SPLIT", "off")
    monkeypatch.setenv("T2V_QTILE", "narrow")
    want = run()
    monkeypatch.setenv("T2V_QTILE", "wide")
    assert all(torch.equal(a, b) for a, b in zip(run(), want))


@pytest.mark.parametrize("lq,lk,H,Hk,D", [([70, 40, 3], [70, 9, 0], 4, 2, 128), ([130, 1], [4000, 50], 3, 1, 64)])
def test_row_statistics_of_the_backward_pass(lq, lk, H, Hk, D):
    """delta_ws as documented, for every row (with no keys, and of cut loops too): -rowsum(dout * out), exact products summed
    in 32 bits, and lse * log2(e), rounded once after log2(e) itself was."""
    log(f"case statistics {lq} over {lk}")
    q, k, v, g = rand(sum(lq), H, D, seed=1), rand(sum(lk), Hk, D, seed=2), rand(sum(lk), Hk, D, seed=3), rand(sum(lq), H, D, seed=4)
    out, lse = t2v.causal_attn_fwd(q, k, v, cu(lq), 0.1, cu_seqlens_k=cu(lk))
    stats = torch.full((2, H, sum(lq)), float("nan"), device="cuda")
    t2v.causal_attn_bwd(q, k, v, out, lse, g, cu(lq), 0.1, delta_ws=stats, cu_seqlens_k=cu(lk))
    torch.cuda.synchronize()
    prod = (out.double() * g.double()).cpu()
    got, want = stats.double().cpu(), -prod.sum(2).t()
    assert ((got[0] - want).abs() <= D * 2.0 ** -24 * prod.abs().sum(2).t()).all()
    scaled = lse.double().cpu() * 1.4426950408889634
    dead = scaled == -float("inf")
    assert torch.equal(dead, got[1] == -float("inf"))
    assert ((got[1] - scaled).abs()[~dead] <= 2.0 ** -23 * scaled.abs()[~dead]).all()


def test_rows_do_not_depend_on_their_neighbours_values():
    """A row's output does not change with other rows' queries, which share its tile and its steps."""
    log("case neighbours")
    H, Hk, D, n = 4, 2, 64, [200]
    q, k, v = rand(200, H, D, seed=1), rand(200, Hk, D, seed=2), rand(200, Hk, D, seed=3)
    a, la = t2v.causal_attn_fwd(q, k, v, cu(n), 0.3)
    q2 = (q * 40).contiguous()
    q2[::7] = q[::7]
    b, lb = t2v.causal_attn_fwd(q2, k, v, cu(n), 0.3)
    torch.cuda.synchronize()
    assert torch.equal(a[::7], b[::7]) and torch.equal(la[:, ::7], lb[:, ::7])


SHAPES = [([300, 65], [300, 65], 6, 2, 128), ([1, 1], [4000, 700], 8, 2, 128), ([40, 500], [900, 500], 3, 1, 64)]


@pytest.mark.parametrize("lq,lk,H,Hk,D", SHAPES)
def test_captured_calls_replay(lq, lk, H, Hk, D):
    """Forward, backward and rotary in a graph, replayed on new inputs with eager calls of other packs between,
    and two graphs in turn."""
    log(f"case capture {lq} {lk} {H}/{Hk}x{D}")
    cq, ck = cu(lq), cu(lk)
    freqs, _ = t2v.rotary_frequencies(16)
    pq, pk = positions(lq), positions(lk)
    st = [rand(sum(lq), H, D, seed=1), rand(sum(lk), Hk, D, seed=2), rand(sum(lk), Hk, D, seed=3), rand(sum(lq), H, D, seed=4)]

    def step():
        q, k, v, g = st
        q2, _ = t2v.rotary_apply(q, None, pq, freqs)
        _, k2 = t2v.rotary_apply(None, k, pk, freqs, "interleaved")
        out, lse = t2v.causal_attn_fwd(q2, k2, v, cq, 0.1, cu_seqlens_k=ck)
        return (out, lse, *t2v.causal_attn_bwd(q2, k2, v, out, lse, g, cq, 0.1, cu_seqlens_k=ck))

    t2v.t2v_release_cache()
    graphs = []
    for _ in range(2):
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=s):
                got = step()
        graphs.append((graph, got))
    for seed in range(5):
        for x, n in zip(st, range(4)):
            x.copy_(rand(*x.shape, seed=10 * seed + n))
        want = [x.clone() for x in step()]
        for i in range(70):  # evicts the lists from the cache
            t2v.causal_attn_fwd(st[0][:1], st[1][:1 + i], st[2][:1 + i], [0, 1], 0.1, cu_seqlens_k=[0, 1 + i])
        for graph, got in graphs:
            graph.replay()
            torch.cuda.synchronize()
            for a, b in zip(got, want):
                assert torch.equal(a, b), seed


def test_captured_autograd():
    """A training step in a graph; and, while an eager graph of the same leaves, made on another stream, is alive, a forward
    pass in one, and the refusal to record a backward pass (it would end the process)."""
    log("case captured autograd")
    n, H, Hk, D = [200, 30], 4, 2, 64
    q, k, v = (rand(230, h, D, seed=h).requires_grad_(True) for h in (H, Hk, Hk))
    g = rand(230, H, D, seed=9)
    pos = positions(n)
    freqs, _ = t2v.rotary_frequencies(32)

    def step():
        q2, k2 = t2v.rotary(q, k, pos, freqs)
        out, _ = t2v.varlen_causal_attention(q2, k2, v, cu(n), 0.1)
        return out

    eager = step()
    want = [x.clone() for x in torch.autograd.grad(eager, (q, k, v), g, retain_graph=True)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        with torch.cuda.graph(forward := torch.cuda.CUDAGraph(), stream=s):
            out = step()
        for leaves in ((q, k, v), (q, k)):  # refused by the attention, which meets v first, and by the rotary positions
            v2 = v if len(leaves) == 3 else v.detach()
            with pytest.raises(RuntimeError, match="eager autograd graph"):
                with torch.cuda.graph(torch.cuda.CUDAGraph(), stream=s):
                    q2, k2 = t2v.rotary(q, k, pos, freqs)
                    torch.autograd.grad(t2v.varlen_causal_attention(q2, k2, v2, cu(n), 0.1)[0], leaves, g)
        forward.replay()
        s.synchronize()
        assert torch.equal(out, eager)
        del out
        again = step()  # eager calls on any stream are fine
        for a, b in zip(torch.autograd.grad(again, (q, k, v), g), want):
            s.synchronize()
            assert torch.equal(a, b)
    del eager, again, q2, k2
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            got = torch.autograd.grad(step(), (q, k, v), g)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
        for a, b in zip(torch.autograd.grad(step(), (q, k, v), g), want):
            torch.cuda.synchronize()
            assert torch.equal(a, b)


def test_second_derivatives():
    """Those of rotary positions, which are linear: of <R x, y> y's. The attention's are refused."""
    log("case second derivatives")
    n = [30]
    x, y = (rand(30, 2, 64, seed=i).requires_grad_(True) for i in (1, 2))
    freqs, _ = t2v.rotary_frequencies(32)
    turned, _ = t2v.rotary(x, None, positions(n), freqs)
    (dx,) = torch.autograd.grad(turned, x, y, create_graph=True)
    w = rand(30, 2, 64, seed=3)
    (dy,) = torch.autograd.grad(dx, y, w)
    torch.cuda.synchronize()
    assert torch.equal(dy, t2v.rotary_apply(w, None, positions(n), freqs)[0])
    out, _ = t2v.varlen_causal_attention(x, x.detach(), x.detach(), cu(n), 0.1)
    (dx,) = torch.autograd.grad(out, x, y, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        dx.float().sum().backward()


def test_other_streams_and_threads():
    """Calls given a stream, and threads with streams of their own, each on packs that no other call uses."""
    log("case streams and threads")
    H, Hk, D = 4, 2, 128
    q, k, v, g = rand(700, H, D, seed=1), rand(700, Hk, D, seed=2), rand(700, Hk, D, seed=3), rand(700, H, D, seed=4)
    torch.cuda.synchronize()

    def all_calls(c, ck, stream):
        tk = int(ck[-1])
        tq = int(c[-1])
        out, lse = t2v.causal_attn_fwd(q[:tq], k[:tk], v[:tk], c, 0.1, stream=stream, cu_seqlens_k=ck)
        return (out, lse, *t2v.causal_attn_bwd(q[:tq], k[:tk], v[:tk], out, lse, g[:tq], c, 0.1, stream=stream,
                                               cu_seqlens_k=ck))

    packs = [(cu([10 * t + i, 3, 1]), cu([600 - 7 * i - t, 30, 5])) for t in range(4) for i in range(20)]
    want = []
    for c, ck in packs:
        want.append([x.clone() for x in all_calls(c, ck, None)])
    torch.cuda.synchronize()
    t2v.t2v_release_cache()
    got, errors = [None] * len(packs), []

    def work(t):
        try:
            s = torch.cuda.Stream()
            for i in range(20):
                got[20 * t + i] = all_calls(*packs[20 * t + i], s)
            s.synchronize()
        except Exception as e:  # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=work, args=(t,)) for t in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        for x, y in zip(a, b):
            assert torch.equal(x, y)


def test_offsets_beyond_32_bits():
    """A cache of 2.6e9 elements: the last sequence gives what it gives alone, forward and backward."""
    log("case long cache")
    Hk, D, tk = 4, 128, 5_000_000
    H = 8
    k = torch.empty((tk, Hk, D), dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    tail = 3000
    k[:-tail] = 0.01
    v[:-tail] = 0.5
    k[-tail:], v[-tail:] = rand(tail, Hk, D, seed=1), rand(tail, Hk, D, seed=2)
    lq, lk = [2, 150], [tk - tail, tail]
    q, g = rand(152, H, D, seed=3), rand(152, H, D, seed=4)
    out, lse = t2v.causal_attn_fwd(q, k, v, cu(lq), 0.1, cu_seqlens_k=cu(lk))
    ref, ref_lse = t2v.causal_attn_fwd(q[2:], k[-tail:].clone(), v[-tail:].clone(), cu([150]), 0.1, cu_seqlens_k=cu([tail]))
    torch.cuda.synchronize()
    r = oracle.causal_attention(q[2:].float().cpu().numpy(), k[-tail:].float().cpu().numpy(), v[-tail:].float().cpu().numpy(),
                                g[2:].float().cpu().numpy(), cu([150]), cu([tail]), 0.1)
    for x in (out[2:], ref):  # the cuts may differ, the results only by rounding
        assert (np.abs(x.double().cpu().numpy() - r["out"]) <= r["bounds"]["out"] + 1e-30).all()
    assert (np.abs(lse[:, 2:].double().cpu().numpy() - r["lse"]) <= r["bounds"]["lse"]).all()
    # equal keys and values: the mean is the value, off by the roundings of P and out; lse = score + ln n
    assert (out[:2].float() - 0.5).abs().max() <= 0.5 * 2.0 ** -8 * 2.02
    score = 0.1 * 0.01 * 1.0 * q[:2].float().sum(2)
    kept = torch.tensor(0.01).bfloat16().float().item() / 0.01
    want = score.t() * kept + torch.log(torch.tensor([tk - tail - 1.0, tk - tail], device="cuda"))
    assert (lse[:, :2] - want).abs().max() <= 1e-3
    dq, dk, dv = t2v.causal_attn_bwd(q, k, v, out, lse, g, cu(lq), 0.1, cu_seqlens_k=cu(lk))
    torch.cuda.synchronize()
    for x, n in ((dq[2:], "dq"), (dk[-tail:], "dk"), (dv[-tail:], "dv")):
        assert (np.abs(x.double().cpu().numpy() - r[n]) <= r["bounds"][n] + 1e-30).all(), n
    del k, v, dk, dv
    torch.cuda.empty_cache()


def test_rows_behind_the_last_sequence_stay():
    log("case larger buffers")
    H, Hk, D = 4, 2, 128
    q, k, v, g = rand(90, H, D, seed=1), rand(200, Hk, D, seed=2), rand(200, Hk, D, seed=3), rand(90, H, D, seed=4)
    full = lambda *s, dtype=torch.bfloat16: torch.full(s, 7.0, dtype=dtype, device="cuda")  # noqa: E731
    out, dq, dk, dv = full(100, H, D), full(100, H, D), full(260, Hk, D), full(260, Hk, D)
    lse = full(H * 90 + 64, dtype=torch.float32)
    c, ck = cu([33, 57]), cu([100, 100])
    t2v.causal_attn_fwd(q, k, v, c, 0.1, out[:90], lse[:H * 90].view(H, 90), cu_seqlens_k=ck)
    t2v.causal_attn_bwd(q, k, v, out[:90], lse[:H * 90].view(H, 90), g, c, 0.1, dq[:90], dk[:200], dv[:200], cu_seqlens_k=ck)
    torch.cuda.synchronize()
    for x, n in ((out, 90), (dq, 90), (dk, 200), (dv, 200), (lse, H * 90)):
        assert (x[n:] == 7.0).all() and not (x[:n] == 7.0).all()


def test_refused_on_the_gpu():
    q, k = rand(9, 4, 64), rand(9, 2, 64)
    for name, kw in (("out", dict(out=rand(8, 4, 64))), ("lse", dict(lse=rand(4, 9)))):
        with pytest.raises(ValueError, match=name):
            t2v.causal_attn_fwd(q, k, k, [0, 9], 0.1, **kw)
    with pytest.raises(ValueError, match="CUDA"):
        t2v.causal_attn_fwd(q, k, k, [0, 9], 0.1, out=rand(9, 4, 64).cpu())
    with pytest.raises(t2v.T2VError, match="multiple"):
        t2v.causal_attn_fwd(rand(9, 3, 64), k, k, [0, 9], 0.1)
    with pytest.raises(t2v.T2VError, match="overlaps"):
        t2v.causal_attn_fwd(q, k, k, [0, 9], 0.1, out=q)
    with pytest.raises(t2v.T2VError, match="overlaps"):
        t2v.rotary_apply(q, None, positions([9]), np.ones(4), q_out=q)
    # offsets in device memory
    host, dev = cu([9]), torch.tensor([0, 9], dtype=torch.int32, device="cuda")
    out, lse = torch.full((9, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((4, 9), 7.0, device="cuda")
    at = lambda x: ctypes.cast(x.data_ptr(), ctypes.POINTER(ctypes.c_int32))  # noqa: E731
    for a, b in ((at(dev), _lib._offsets_ptr(host)), (_lib._offsets_ptr(host), at(dev))):
        st = _lib.lib().t2v_causal_fwd(q.data_ptr(), k.data_ptr(), k.data_ptr(), 256, 128, 128, a, b, 1, 4, 2, 64, 0.1,
                                       out.data_ptr(), lse.data_ptr(), None, 0, None, None)
        assert st == _lib.T2V_ERR_INVALID_ARG and "host pointer" in _lib.t2v_last_error()
    # a workspace that is too small: nothing is launched
    k = rand(4000, 2, 64)
    need = ctypes.c_uint64(0)
    c1, c2 = cu([1]), cu([4000])
    args = (q.data_ptr(), k.data_ptr(), k.data_ptr(), 256, 128, 128, _lib._offsets_ptr(c1), _lib._offsets_ptr(c2), 1, 4, 2, 64,
            0.1, out.data_ptr(), lse.data_ptr())
    assert _lib.lib().t2v_causal_fwd(*args, None, 0, ctypes.byref(need), None) == _lib.T2V_ERR_WORKSPACE and need.value > 0
    ws = torch.empty(need.value, dtype=torch.uint8, device="cuda")
    st = _lib.lib().t2v_causal_fwd(*args, ws.data_ptr(), need.value - 1, ctypes.byref(need), None)
    torch.cuda.synchronize()
    assert st == _lib.T2V_ERR_WORKSPACE and (out == 7.0).all() and (lse == 7.0).all()
    assert _lib.lib().t2v_causal_fwd(*args, ws.data_ptr(), need.value, ctypes.byref(need), None) == _lib.T2V_OK
    torch.cuda.synchronize()
    assert torch.isfinite(out[0].float()).all() and (out[1:] == 7.0).all()
