"""Pages handed out, shared, copied on write, freed and compacted, on the CPU, against sequences kept as lists; and the refusals of the
paged calls: by the C ABI (fake addresses, never dereferenced) and by the binding."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2607_01701_amd as t2v
from paper_2607_01701_amd import _lib
from paper_2607_01701_amd.page_table import PageTable

A, MB = 0x100000, 1 << 20
INV, UNS, WS = _lib.T2V_ERR_INVALID_ARG, _lib.T2V_ERR_UNSUPPORTED, _lib.T2V_ERR_WORKSPACE


class Memory:
    """What the GPU would hold: rows of pages, copied as the table says before tokens are written."""

    def __init__(self, pages, page_size, sequences, width):
        self.t = PageTable(pages, page_size, sequences, width)
        self.rows = np.full((pages, page_size), -1, dtype=np.int64)

    def copy(self, pairs):
        src, dst = pairs
        assert np.unique(dst).size == dst.size and not set(src.tolist()) & set(dst.tolist())
        self.rows[dst] = self.rows[src]

    def write(self, s, first, values):
        for i, x in enumerate(values):
            j, r = divmod(first + i, self.t.page_size)
            assert self.t.refs[self.t.table[s, j]] == 1  # nobody else's
            self.rows[self.t.table[s, j], r] = x

    def read(self, s):
        n, p = int(self.t.lengths[s]), self.t.page_size
        return [int(self.rows[self.t.table[s, j // p], j % p]) for j in range(n)]

    def check(self, model):
        t = self.t
        for s in range(t.active.size):
            assert bool(t.active[s]) == (s in model)
            assert self.read(s) == model.get(s, [])
            assert (t.table[s, t.counts[s]:] == -1).all() and (t.table[s, :t.counts[s]] >= 0).all()
        refs = np.bincount(t.table[t.table >= 0], minlength=t.refs.size)
        assert (refs == t.refs).all()
        assert sorted(t._free) == np.flatnonzero(t.refs == 0).tolist()


@pytest.mark.parametrize("seed", range(12))
def test_random_lives(seed):
    r = np.random.default_rng(seed)
    m = Memory(40, 16, 9, 12)
    model, value = {}, 0
    for _ in range(400):
        do = r.integers(0, 8)
        live = list(model)
        before = (m.t.table.copy(), m.t.lengths.copy(), m.t.refs.copy(), m.t.counts.copy())
        try:
            if do == 0:
                model[m.t.add()] = []
            elif do in (1, 2, 3) and live:
                some = r.permutation(live)[:r.integers(1, len(live) + 1)]
                more = r.integers(0, [3, 40][r.integers(2)], some.size)
                if r.random() < 0.3:  # a captured step: room first, tokens one by one
                    m.copy(m.t.reserve(some, more))
                    more = np.minimum(more, r.integers(0, 40, some.size))
                    first = m.t.lengths.copy()
                    m.t.grown(some, more)
                else:
                    first = m.t.lengths.copy()
                    m.copy(m.t.extend(some, more))
                for s, n in zip(some.tolist(), more.tolist()):
                    new = list(range(value, value + n))
                    value += n
                    m.write(s, int(first[s]), new)
                    model[s] += new
            elif do == 4 and live:
                s = int(r.choice(live))
                model[m.t.fork(s)] = list(model[s])
            elif do == 5 and live:
                s = int(r.choice(live))
                m.t.free(s)
                del model[s]
            elif do == 6 and live:
                s = int(r.choice(live))
                n = int(r.integers(0, len(model[s]) + 1))
                m.t.truncate(s, n)
                model[s] = model[s][:n]
            elif do == 7:
                m.copy(m.t.compact())
                used = int((m.t.refs > 0).sum())
                assert (m.t.refs[:used] > 0).all()
        except RuntimeError as e:  # no pages, no sequence, too long: nothing has changed
            assert "pages" in str(e) or "in use" in str(e)
            assert all((a == b).all() for a, b in zip(before, (m.t.table, m.t.lengths, m.t.refs, m.t.counts)))
        m.check(model)


def test_forks_share_full_pages_and_copy_the_begun_one():
    m = Memory(10, 16, 4, 8)
    s = m.t.add()
    m.copy(m.t.extend([s], [40]))
    m.write(s, 0, range(40))
    f = m.t.fork(s)
    assert m.t.free_pages == 7 and (m.t.table[f, :3] == m.t.table[s, :3]).all()
    src, dst = m.t.extend([s, f], [1, 1])
    assert src.tolist() == [int(m.t.table[f, 2])] and dst.tolist() == [int(m.t.table[s, 2])]  # the last to be seen keeps it
    assert (m.t.table[f, :2] == m.t.table[s, :2]).all() and m.t.free_pages == 6
    m.t.free(s)
    assert m.t.free_pages == 7


@pytest.mark.parametrize("do,err,msg", [
    (lambda t: t.extend([0, 0], [1, 1]), ValueError, "different"), (lambda t: t.extend([3], [1]), ValueError, "not in use"),
    (lambda t: t.extend([9], [1]), ValueError, "not in use"), (lambda t: t.extend([-1], [1]), ValueError, "not in use"),
    (lambda t: t.extend([0], [-1]), ValueError, ">= 0"), (lambda t: t.extend([0], [1.5]), ValueError, "whole"),
    (lambda t: t.extend([0.0], [1]), ValueError, "whole"), (lambda t: t.extend([0], [2 ** 31]), ValueError, "whole"),
    (lambda t: t.extend([0], [1000]), RuntimeError, "passes its"),
    (lambda t: t.extend([0], [90]), RuntimeError, "pages are needed"), (lambda t: t.grown([0], [16]), ValueError, "reserved"),
    (lambda t: t.fork(2), ValueError, "not in use"), (lambda t: t.free(2), ValueError, "not in use"),
    (lambda t: t.truncate(0, 9), ValueError, "tokens"), (lambda t: PageTable(4, 24, 1, 1), ValueError, "power of two"),
    (lambda t: PageTable(4, 16, 0, 1), ValueError, "at least"), (lambda t: [t.add() for _ in range(4)], RuntimeError, "in use"),
])
def test_page_table_refusals(do, err, msg):
    t = PageTable(5, 16, 4, 10)
    t.add()
    t.extend([0], [8])
    with pytest.raises(err, match=msg):
        do(t)
    assert t.lengths.tolist() == [8, 0, 0, 0] and t.free_pages == 4


def test_forks_and_truncations_end_reserved_room():
    m = Memory(10, 16, 4, 8)
    s = m.t.add()
    m.copy(m.t.extend([s], [20]))
    m.write(s, 0, range(20))
    m.copy(m.t.reserve([s], 9))
    m.t.grown([s], 4)
    m.write(s, 20, range(20, 24))
    with pytest.raises(ValueError, match="reserved"):
        m.t.grown([s], 6)
    f = m.t.fork(s)  # the next tokens of s would go to a page that f has
    for x in (s, f):
        with pytest.raises(ValueError, match="reserved"):
            m.t.grown([x], 1)
    src, _ = m.t.reserve([s], 2)
    assert src.tolist() == [int(m.t.table[f, 1])]
    m.t.grown([s], 1)
    m.t.truncate(s, 10)
    with pytest.raises(ValueError, match="reserved"):
        m.t.grown([s], 1)
    assert m.t.lengths[[s, f]].tolist() == [10, 24]


# ------------------------------------------------------------------------ the calls


def cache(**kw):
    p = dict(k=A, v=A + 64 * MB, ks=(16 * 256, 256, 128), vs=(16 * 256, 256, 128), pages=100, table=A + 128 * MB, stride=7, width=7,
             lengths=A + 129 * MB, nseq=3, page=16, hk=2, d=128)
    p.update(kw)
    i3 = ctypes.c_int64 * 3
    return _lib.PagesStruct(p["k"], p["v"], i3(*p["ks"]), i3(*p["vs"]), p["pages"], p["table"], p["stride"], p["width"], p["lengths"],
                            p["nseq"], p["page"], p["hk"], p["d"])


def call(which, c=None, **kw):
    p = dict(q=A + 192 * MB, qs=768, heads=6, cu=A + 130 * MB, tokens=9, scale=0.1, out=A + 256 * MB, lse=A + 320 * MB,
             ws=A + 384 * MB, ws_bytes=200 * MB, kn=A + 640 * MB, vn=A + 704 * MB, ksn=256, vsn=256, turn=True)
    p.update(kw)
    L, need = _lib.lib(), ctypes.c_uint64(7)
    ref = None if c == "none" else ctypes.byref(cache(**(c or {})))
    if which == "attn":
        st = L.t2v_paged_fwd(p["q"], p["qs"], p["heads"], p["cu"], p["tokens"], ref, p["scale"], p["out"], p["lse"], p["ws"],
                             p["ws_bytes"], ctypes.byref(need), None)
    else:
        t = _lib.Turn()
        t.eps = 1e-6
        st = L.t2v_paged_append(p["kn"], p["vn"], p["ksn"], p["vsn"], p["q"], p["qs"], p["heads"], p["cu"], p["tokens"], ref,
                                ctypes.byref(t) if p["turn"] else None, p["out"], None)
    return st, _lib.t2v_last_error(L), need.value


CACHES = [
    ({"d": 96}, UNS, "head_dim"), ({"hk": 0}, INV, "kv_heads"), ({"hk": 1 << 20}, INV, "kv_heads"), ({"page": 8}, INV, "page_size"),
    ({"page": 48}, INV, "page_size"), ({"page": 1 << 17}, INV, "page_size"), ({"pages": -1}, INV, "pages"), ({"pages": 1 << 31}, INV, "pages"),
    ({"nseq": -1}, INV, "nseq"), ({"width": -1}, INV, "width"), ({"width": 1 << 27}, INV, "width"), ({"stride": 6}, INV, "table_stride"),
    ({"ks": (4096, 252, 128)}, INV, "k_strides"), ({"ks": (4096, 256, 120)}, INV, "overlap"), ({"vs": (4096, 128, 128)}, INV, "v_strides let rows"),
    ({"vs": (4088, 256, 128)}, INV, "v_strides let pages"), ({"ks": (-4096, 256, 128)}, INV, "k_strides"), ({"ks": (1 << 41, 256, 128)}, INV, "large"),
    ({"k": 0}, INV, "cache.k is NULL"), ({"v": A + 8}, INV, "cache.v is not"), ({"lengths": 0}, INV, "lengths is NULL"),
    ({"table": 0}, INV, "table is NULL"), ({"table": A + 2}, INV, "table is not"),
]


@pytest.mark.parametrize("which", ["attn", "append"])
@pytest.mark.parametrize("kw,status,msg", CACHES)
def test_cache_refusals(which, kw, status, msg):
    st, err, _ = call(which, kw)
    assert st == status and msg in err, (st, err)


@pytest.mark.parametrize("which,kw,status,msg", [
    ("attn", {"heads": 5}, INV, "multiple"), ("attn", {"heads": 0}, INV, "multiple"), ("attn", {"scale": float("inf")}, INV, "scale"),
    ("attn", {"tokens": -1}, INV, "tokens"), ("attn", {"tokens": 1 << 30}, INV, "tokens"),
    ("attn", {"qs": 760}, INV, "q_stride"), ("attn", {"q": 0}, INV, "q is NULL"), ("attn", {"cu": 0}, INV, "cu_seqlens is NULL"),
    ("attn", {"cu": A + 1}, INV, "cu_seqlens is not"), ("attn", {"out": A + 4096}, INV, "out overlaps input cache.k"),
    ("attn", {"out": A + 130 * MB - 16}, INV, "cu_seqlens"), ("attn", {"lse": A + 129 * MB}, INV, "lengths"),
    ("attn", {"ws": A + 128 * MB}, INV, "overlaps"), ("attn", {"ws_bytes": 64}, WS, "workspace"), ("attn", {"ws": 0, "ws_bytes": 0}, WS, "needs"),
    ("attn", {"lse": A + 256 * MB}, INV, "overlaps"),
    ("append", {"heads": -1}, INV, "heads"), ("append", {"turn": False}, INV, "without a norm"), ("append", {"ksn": 248}, INV, "k_stride"),
    ("append", {"vsn": 260}, INV, "v_stride"), ("append", {"qs": 0}, INV, "q_stride"), ("append", {"kn": A + 4096}, INV, "overlaps input k"),
    ("append", {"vn": A + 64 * MB}, INV, "overlaps input v"), ("append", {"out": A + 192 * MB}, INV, "q_out overlaps"),
    ("append", {"cu": A + 16}, INV, "cu_seqlens"), ("append", {"tokens": -1}, INV, "tokens"), ("append", {"vn": 0}, INV, "v is NULL"),
])
def test_call_refusals(which, kw, status, msg):
    st, err, need = call(which, **kw)
    assert st == status and msg in err, (st, err)
    assert which == "append" or (need > 0) == (status == WS)


def test_more_refusals():
    assert call("append", {"v": A})[0] == INV
    assert call("attn", "none")[0] == INV and call("append", "none")[0] == INV
    st, err, _ = call("attn", {"width": 1 << 26, "stride": 1 << 26}, tokens=1 << 28, heads=2, qs=256)
    assert st == INV, err
    # the workspace that a call asks for follows from its sizes and stays below what is documented
    for d, hk, heads in ((128, 2, 6), (64, 2, 6), (128, 2, 32)):
        _, _, need = call("attn", {"d": d, "hk": hk, "width": 4096, "stride": 4096, "nseq": 64}, tokens=4000, heads=heads, qs=heads * d, ws_bytes=0, ws=0)
        assert 0 < need <= 72 * MB


def test_empty_calls():
    none = dict(q=None, cu=None, out=None, lse=None, ws=None, ws_bytes=0, kn=None, vn=None)
    for which in ("attn", "append"):
        assert call(which, tokens=0, **none)[0] == _lib.T2V_OK
        assert call(which, {"nseq": 0, "table": None, "lengths": None}, **none)[0] == _lib.T2V_OK


def copy(**kw):
    p = dict(buffers=[A, A + 64 * MB], pages=10, stride=4096, bytes=4096, src=[1, 2], dst=[3, 4])
    p.update(kw)
    b = None if p["buffers"] is None else (ctypes.c_void_p * len(p["buffers"]))(*p["buffers"])
    i = [None if x is None else np.ascontiguousarray(x, dtype=np.int32) for x in (p["src"], p["dst"])]
    L = _lib.lib()
    st = L.t2v_page_copy(b, p.get("n_buffers", 0 if b is None else len(b)), p["pages"], p["stride"], p["bytes"],
                         *(None if x is None else x.ctypes.data for x in i), p.get("n", 0 if i[0] is None else len(i[0])), None)
    return st, _lib.t2v_last_error(L)


@pytest.mark.parametrize("kw,msg", [
    ({"src": [10, 2]}, "outside"), ({"dst": [-1, 2]}, "outside"), ({"dst": [3, 3]}, "written twice"), ({"dst": [3, 1]}, "both read"),
    ({"src": [3, 2]}, "both read"), ({"bytes": 4100}, "multiples"), ({"bytes": 0}, "multiples"), ({"stride": 4080}, "multiples"),
    ({"buffers": [A, 0]}, "NULL"), ({"buffers": [A, A + 8]}, "aligned"), ({"pages": -1}, "pages"), ({"n": -1}, "n must be"),
    ({"src": None, "n": 2}, "NULL"), ({"buffers": None, "n_buffers": 1}, "NULL"), ({"n_buffers": -1}, "n_buffers"),
    ({"bytes": 1 << 40, "stride": 1 << 40}, "too large"),
])
def test_page_copy_refusals(kw, msg):
    st, err = copy(**kw)
    assert st == INV and msg in err, (st, err)


def test_page_copy_of_nothing():
    assert copy(src=[], dst=[])[0] == _lib.T2V_OK and copy(buffers=[])[0] == _lib.T2V_OK
    t2v.page_copy([], [], [])


def _t(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


@pytest.mark.parametrize("kw", [{"src": np.array([2 ** 32])}, {"dst": [1.0]}, {"src": [True]}, {"dst": np.array([-2 ** 31 - 1])}])
def test_page_copy_takes_no_other_numbers(kw):
    a = dict(src=[1], dst=[2])
    a.update(kw)
    with pytest.raises(ValueError, match="page numbers"):
        t2v.page_copy(_t(4, 16, 8), a["src"], a["dst"])


@pytest.mark.parametrize("kw,msg", [
    ({"src": [1], "dst": [2, 3]}, "one length"), ({"src": [[1]], "dst": [[2]]}, "1-D"), ({"buffers": [_t(4, 16, 8), _t(4, 16, 9)]}, "one shape"),
    ({"buffers": [_t(4, 16, 8), _t(4, 16, 8, dtype=torch.float32)]}, "one shape"), ({"buffers": _t(4, 16, 16)[..., ::2]}, "dense"),
    ({"buffers": _t(4)}, "pages"), ({"buffers": _t(4, 0)}, "pages"), ({}, "CUDA"), ({"buffers": _t(4, 2, 16, 8).transpose(1, 2)}, "CUDA"),
])
def test_page_copy_binding_refusals(kw, msg):
    a = dict(buffers=_t(4, 16, 8), src=[1], dst=[2])
    a.update(kw)
    with pytest.raises(ValueError, match=msg):
        t2v.page_copy(a["buffers"], a["src"], a["dst"])


@pytest.mark.parametrize("kw,msg", [
    ({"k": _t(4, 16, 256)}, "k must be"), ({"v": _t(4, 16, 2, 64)}, "v has shape"), ({"k": _t(4, 16, 2, 128, dtype=torch.float16)}, "dtype"),
    ({"v": _t(4, 16, 2, 256)[..., ::2]}, "contiguously"), ({"table": _t(3, 5)}, "table"), ({"table": _t(5, 3, dtype=torch.int32).t()}, "table"),
    ({"lengths": _t(4, dtype=torch.int32)}, "lengths"), ({"lengths": _t(3, dtype=torch.int64)}, "lengths"), ({}, "CUDA"),
])
def test_pages_refusals(kw, msg):
    a = dict(k=_t(4, 16, 2, 128), v=_t(4, 16, 2, 128), table=_t(3, 5, dtype=torch.int32), lengths=_t(3, dtype=torch.int32))
    a.update(kw)
    with pytest.raises(ValueError, match=msg):
        t2v.Pages(**a)


@pytest.fixture
def pages(monkeypatch):
    monkeypatch.setattr(_lib, "_check_on_device", lambda named: None)
    p = t2v.Pages(_t(4, 16, 2, 128), _t(4, 16, 2, 128), _t(3, 5, dtype=torch.int32), _t(3, dtype=torch.int32))
    monkeypatch.undo()
    p.device = torch.device("cuda", 0)  # as pages have
    return p


@pytest.mark.parametrize("kw,msg", [
    ({"q": _t(9, 768)}, "head_dim"), ({"q": _t(9, 6, 64)}, "head_dim"), ({"q": _t(9, 6, 128, dtype=torch.float32)}, "dtype"),
    ({"cu": _t(3, dtype=torch.int32)}, "cu_seqlens"), ({"cu": _t(4, dtype=torch.int64)}, "cu_seqlens"), ({}, "CUDA"),
])
def test_attention_binding_refusals(pages, kw, msg):
    a = dict(q=_t(9, 6, 128), cu=_t(4, dtype=torch.int32))
    a.update(kw)
    with pytest.raises(ValueError, match=msg):
        t2v.paged_attn_fwd(a["q"], pages, a["cu"], 0.1)


@pytest.mark.parametrize("kw,msg", [
    ({"k": _t(9, 256)}, "head_dim"), ({"k": _t(9, 3, 128)}, "k has shape"), ({"v": _t(8, 2, 128)}, "v has shape"),
    ({"q": _t(9, 6, 128)}, "without a norm"), ({"positions": _t(9, dtype=torch.int32)}, "without a norm"),
    ({"q": _t(8, 6, 128), "eps": 1e-6}, "q has shape"), ({"q_out": _t(9, 6, 128)}, "q_out is given"), ({"freqs": np.ones(4)}, "positions"),
    ({"eps": -1.0}, "eps"), ({"eps": 1e-6, "k_weight": _t(64)}, "k_weight"), ({}, "CUDA"),
])
def test_append_binding_refusals(pages, kw, msg):
    a = dict(k=_t(9, 2, 128), v=_t(9, 2, 128), cu_seqlens=_t(4, dtype=torch.int32))
    a.update(kw)
    with pytest.raises(ValueError, match=msg):
        t2v.paged_append(a.pop("k"), a.pop("v"), pages, a.pop("cu_seqlens"), **a)
