"""Attention over a paged cache on the GPU against the float64 oracle with its bounds: single tokens, chunks, prompts and mixtures,
every page size, both layouts of a page, empty rows, pages and lengths that no cache has, growing lengths in captured graphs."""
import numpy as np
import pytest
import torch

from oracle import causal_attention
from paper_2607_01701_amd import Pages, causal_attn_fwd, paged_attn_fwd, use_checked_library

from gpu_util import log
from paged_util import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def np64(x):
    return x.detach().double().cpu().numpy()


def reference(c):
    n = sum(c.queries)
    cu_q = np.concatenate([[0], np.cumsum(c.queries)])
    return causal_attention(np64(c.q[:n]), np64(c.k), np64(c.v), None, cu_q, c.cu_k, c.scale)


def check(c, out, lse, ref=None):
    n = sum(c.queries)
    ref = reference(c) if ref is None else ref
    e = np.abs(np64(out[:n]) - ref["out"])
    worst = float((e / (ref["bounds"]["out"] + 1e-300)).max()) if e.size else 0.0
    got = np64(lse[:, :n])
    empty = np.isneginf(ref["lse"])
    assert (np.isneginf(got) == empty).all()
    d = np.abs(np.where(empty, 0.0, got) - np.where(empty, 0.0, ref["lse"]))
    worst_lse = float((d / (ref["bounds"]["lse"] + 1e-300)).max()) if d.size else 0.0
    log(f"  out {worst:.3f}, lse {worst_lse:.3f} of the bound")
    assert worst <= 1.0 and worst_lse <= 1.0
    assert (np64(out[:n])[np.moveaxis(empty, 0, 1)] == 0).all()


CASES = [  # H, Hk, D, page, queries, keys
    (40, 8, 128, 64, [1], [1]), (30, 10, 64, 16, [1], [1280]), (8, 2, 128, 16, [1] * 6, [1, 15, 16, 17, 300, 33]),
    (6, 2, 64, 32, [1, 2, 4, 3], [64, 65, 127, 1000]), (3, 1, 128, 128, [1] * 5, [127, 128, 129, 255, 2000]),
    (16, 1, 64, 256, [1, 1, 2], [700, 256, 257]), (12, 4, 128, 32, [77, 130], [77, 600]), (24, 8, 128, 16, [45], [45]),
    (4, 4, 64, 16, [200, 129, 64], [200, 400, 65]), (2, 1, 64, 64, [300], [300]), (6, 2, 128, 64, [1, 50, 1, 1, 33, 0, 2], [900, 50, 64, 31, 1000, 40, 5]),
    (40, 1, 128, 16, [1, 3, 20], [500, 40, 60]), (5, 1, 128, 64, [7, 26], [7, 700]), (1, 1, 128, 16, [1, 33, 129], [2500, 33, 129]),
    (12, 4, 128, 64, [5, 3, 0, 1, 40], [3, 0, 10, 0, 17]),  # queries without keys, fewer keys than queries
    (7, 7, 64, 1024, [1, 12], [1500, 1100]), (64, 2, 64, 16, [1, 1], [129, 1000]),
]


@pytest.mark.parametrize("heads_first", [False, True], ids=["tokens", "heads"])
@pytest.mark.parametrize("H,Hk,D,page,queries,keys", CASES)
def test_values(H, Hk, D, page, queries, keys, heads_first):
    log(f"case {H}/{Hk}x{D} page {page} {queries} over {keys} heads first {heads_first}")
    c = Case(H, Hk, D, page, queries, keys, heads_first=heads_first)
    ref = reference(c)
    check(c, *paged_attn_fwd(c.q, c.pages, c.cu, c.scale), ref)


@pytest.mark.parametrize("H,Hk,D,page,queries,keys", [
    (3, 1, 128, 64, [1], [20000]), (1, 1, 64, 16, [1], [9000]), (32, 1, 128, 64, [1], [9000]), (5, 1, 64, 64, [3], [12000]),  # tiles of many pieces
    (24, 8, 128, 64, [1], [300]), (8, 2, 64, 16, [1] * 3, [129, 500, 40]), (12, 4, 128, 64, [64], [500]), (6, 2, 128, 32, [1, 40], [700, 300]),
])
def test_wide_tables_and_many_pieces(H, Hk, D, page, queries, keys):
    log(f"case {H} {Hk} {D} {page} {queries} {keys}")
    c = Case(H, Hk, D, page, queries, keys, width=3000)  # room for far more than there is: few workgroups get a share
    check(c, *paged_attn_fwd(c.q, c.pages, c.cu, c.scale))


def test_many_sequences():
    log("case many sequences")
    r = np.random.default_rng(0)
    for n, kind in ((200, "tokens"), (65, "mixed"), (64, "tokens"), (129, "mixed")):
        keys = r.integers(0, 200, n).tolist()
        queries = [int(min(k, 1)) if kind == "tokens" or r.random() < 0.8 else int(r.integers(0, k + 1)) for k in keys]
        c = Case(4, 2, 64, 16, queries, keys, seed=n)
        check(c, *paged_attn_fwd(c.q, c.pages, c.cu, c.scale))


def test_random_batches():
    r = np.random.default_rng(1)
    for i in range(25):
        H, Hk, D = [(2, 1, 64), (6, 2, 64), (4, 4, 128), (12, 2, 128), (5, 1, 64), (16, 1, 128)][r.integers(6)]
        n = int(r.integers(1, 12))
        keys = [int(np.exp(r.uniform(0, np.log(900)))) for _ in range(n)]
        queries = [int(r.integers(0, min(k + 2, 3)) if r.random() < 0.6 else r.integers(0, k + 1)) for k in keys]
        page = int(2 ** r.integers(4, 9))
        log(f"case random {i}: {H}/{Hk}x{D} page {page} {queries} over {keys}")
        c = Case(H, Hk, D, page, queries, keys, seed=i, heads_first=bool(r.integers(2)), fused=bool(r.integers(2)))
        check(c, *paged_attn_fwd(c.q, c.pages, c.cu, c.scale))


@pytest.mark.parametrize("scale", [0.0, -0.2, 3.0, 1e-4])
def test_scales_and_slices(scale):
    log(f"case scale {scale}")
    for queries, keys in (([1, 1], [300, 50]), ([60], [200])):
        c = Case(6, 2, 64, 16, queries, keys, scale=scale, fused=True)
        check(c, *paged_attn_fwd(c.q, c.pages, c.cu, c.scale))


def test_rows_behind_the_last_sequence_stay():
    log("case padding")
    for queries, keys in (([1, 1, 0], [300, 50, 0]), ([60, 1], [200, 9])):
        c = Case(6, 2, 128, 16, queries, keys, extra_rows=5)
        c.q[sum(queries):] = float("nan")
        out = torch.full((c.T, 6, 128), 7.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((6, c.T), 7.0, device="cuda")
        paged_attn_fwd(c.q, c.pages, c.cu, c.scale, out=out, lse=lse)
        check(c, out, lse)
        assert (out[sum(queries):] == 7.0).all() and (lse[:, sum(queries):] == 7.0).all()


def test_infinities_and_nan_stay_behind_the_mask():
    log("case odd values")
    for queries, keys in (([4, 40], [40, 300]), ([4], [40])):
        c = Case(6, 2, 128, 16, queries, keys)
        clean, clean_lse = paged_attn_fwd(c.q, c.pages, c.cu, c.scale)
        p, r = c.slots[0]
        c.pages.v[p[-1], r[-1], 0, 3] = float("inf")  # the last key, seen by the last query only
        c.pages.k[p[-2], r[-2], 1, 5] = float("nan")  # seen by the last two
        out, lse = paged_attn_fwd(c.q, c.pages, c.cu, c.scale)
        torch.cuda.synchronize()
        same = torch.ones(sum(queries), 6, dtype=torch.bool)
        same[3, :3] = False
        same[2:4, 3:] = False
        assert torch.equal(out[same], clean[same]) and torch.equal(lse.t()[same], clean_lse.t()[same])
        assert out[3, :3, 3].isinf().all() and out[2:4, 3:].isnan().all() and lse[3:, 2:4].isnan().all()


@pytest.mark.parametrize("bad", [-1, 10 ** 6, 2 ** 31 - 1, -2 ** 31])
def test_pages_outside_the_cache_give_nan_where_they_are_seen(bad):
    log(f"case bad page {bad}")
    # (a) tokens: one sequence reads the page, the others do not
    c = Case(6, 2, 128, 16, [1, 1, 1], [100, 40, 300])
    clean, clean_lse = paged_attn_fwd(c.q, c.pages, c.cu, c.scale)
    c.pages.table[2, 7] = bad
    out, lse = paged_attn_fwd(c.q, c.pages, c.cu, c.scale)
    assert torch.equal(out[:2], clean[:2]) and torch.equal(lse[:, :2], clean_lse[:, :2])
    assert out[2].isnan().all() and lse[:, 2].isnan().all()
    # (b) a prompt: queries before the page's keys do not see it
    c = Case(6, 2, 64, 16, [90], [90])
    clean, clean_lse = paged_attn_fwd(c.q, c.pages, c.cu, c.scale)
    c.pages.table[0, 3] = bad
    out, lse = paged_attn_fwd(c.q, c.pages, c.cu, c.scale)
    assert torch.equal(out[:48], clean[:48]) and torch.equal(lse[:, :48], clean_lse[:, :48])
    assert out[48:].isnan().all() and lse[:, 48:].isnan().all()


def test_lengths_beyond_the_table_give_nan():
    log("case long lengths")
    for queries in ([1, 1, 1], [1, 40, 1]):
        c = Case(6, 2, 128, 16, queries, [100, 60, 30], width=7)
        clean, clean_lse = paged_attn_fwd(c.q, c.pages, c.cu, c.scale)
        for length in (113, 2 ** 31 - 1):
            c.pages.lengths[0] = length
            c.pages.lengths[2] = -2 ** 31
            out, lse = paged_attn_fwd(c.q, c.pages, c.cu, c.scale)
            assert out[0].isnan().all() and lse[:, 0].isnan().all()
            assert (out[-1] == 0).all() and lse[:, -1].isneginf().all()
            assert torch.equal(out[1:-1], clean[1:-1]) and torch.equal(lse[:, 1:-1], clean_lse[:, 1:-1])


def test_offsets_that_no_batch_has_touch_nothing_outside():
    log("case offsets")
    c = Case(4, 2, 64, 16, [3, 2, 4], [30, 20, 40])
    buf = torch.full((c.T + 64, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((4, c.T), 7.0, device="cuda")
    for cu in ([0, 5, 2, 9], [-5, 3, 1000, 2000], [9, 9, 9, 9], [2 ** 31 - 1, -2 ** 31, 0, 4], [0, 0, 0, 0]):
        paged_attn_fwd(c.q, c.pages, torch.tensor(cu, dtype=torch.int32, device="cuda"), c.scale, out=buf[32:32 + c.T], lse=lse)
        torch.cuda.synchronize()
        assert (buf[:32] == 7.0).all() and (buf[32 + c.T:] == 7.0).all()


def test_offsets_that_multiply_the_work_end_without_any():
    log("case many long sequences with the queries of one")
    n, T, width = 4096, 8192, 16384
    k = torch.ones(1, 65536, 1, 64, dtype=torch.bfloat16, device="cuda")
    pages = Pages(k, k.clone(), torch.zeros(n, width, dtype=torch.int32, device="cuda"), torch.full((n,), 2 ** 30, dtype=torch.int32, device="cuda"))
    cu = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
    cu[1::2] = T
    q = torch.zeros(T, 16, 64, dtype=torch.bfloat16, device="cuda")
    out = torch.full_like(q, 7.0)
    paged_attn_fwd(q, pages, cu, 0.1, out=out)
    torch.cuda.synchronize()
    assert (out == 7.0).all()


def test_no_queries_no_sequences():
    c = Case(4, 2, 64, 16, [0, 0], [30, 20])
    out, lse = paged_attn_fwd(c.q, c.pages, c.cu, c.scale)
    assert out.shape == (0, 4, 64) and lse.shape == (4, 0)
    e = Pages(c.pages.k, c.pages.v, c.pages.table[:0], c.pages.lengths[:0])
    out = torch.full((3, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    paged_attn_fwd(out.clone(), e, torch.zeros(1, dtype=torch.int32, device="cuda"), 0.1, out=out)
    assert (out == 7.0).all()
    n = Pages(c.pages.k[:0], c.pages.v[:0], c.pages.table[:, :0], torch.zeros(2, dtype=torch.int32, device="cuda"))
    out, lse = paged_attn_fwd(torch.ones(2, 4, 64, dtype=torch.bfloat16, device="cuda"), n,
                              torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda"), 0.1)
    assert (out == 0).all() and lse.isneginf().all()


def test_strides_of_interleaved_caches():
    """K and V of a layer as slices of one tensor [pages, layers, 2, page_size, Hk, D], and table rows with room between."""
    log("case interleaved")
    c = Case(6, 2, 64, 16, [1, 20], [100, 90])
    ref = paged_attn_fwd(c.q, c.pages, c.cu, c.scale)
    n = c.pages.k.shape[0]
    whole = torch.full((n, 3, 2, 16, 2, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    whole[:, 1, 0], whole[:, 1, 1] = c.pages.k, c.pages.v
    table = torch.full((2, 50), -1, dtype=torch.int32, device="cuda")
    w = c.pages.table.shape[1]
    table[:, :w] = c.pages.table
    got = paged_attn_fwd(c.q, Pages(whole[:, 1, 0], whole[:, 1, 1], table[:, :w], c.pages.lengths), c.cu, c.scale)
    assert all(torch.equal(a, b) for a, b in zip(got, ref))


def test_a_cache_beyond_32_bit_offsets():
    log("case large cache")
    page, Hk, D = 64, 8, 128
    n = 40_000  # 5.2 GB of keys: 2.6e9 elements
    k = torch.empty(n, page, Hk, D, dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    at = [n - 1, 0, n - 2, n // 2 + 17]
    small_k, small_v = (torch.randn(4, page, Hk, D, device="cuda").bfloat16() for _ in range(2))
    k[at], v[at] = small_k, small_v
    cu = torch.tensor([0, 1, 41], dtype=torch.int32, device="cuda")
    q = torch.randn(41, 24, D, device="cuda").bfloat16()
    lengths = torch.tensor([250, 199], dtype=torch.int32, device="cuda")
    table = torch.tensor([at, at], dtype=torch.int32, device="cuda")
    got = paged_attn_fwd(q, Pages(k, v, table, lengths), cu, 0.1)
    few = torch.tensor([[0, 1, 2, 3]] * 2, dtype=torch.int32, device="cuda")
    ref = paged_attn_fwd(q, Pages(small_k, small_v, few, lengths), cu, 0.1)
    assert all(torch.equal(a, b) for a, b in zip(got, ref)) and got[0].isfinite().all()


def test_against_the_packed_call():
    """Long loops, cut in many pieces, against causal_attn_fwd, which is tested by itself: twice the bound of one rounding."""
    log("case packed")
    for H, Hk, D, queries, keys in ((40, 8, 128, [1] * 4, [20280, 31, 7000, 2051]), (12, 4, 128, [768, 257], [9000, 4097]),
                                    (30, 10, 64, [1500, 1, 40], [1500, 8191, 4000])):
        c = Case(H, Hk, D, 64, queries, keys)
        got, lse = paged_attn_fwd(c.q, c.pages, c.cu, c.scale)
        ref, ref_lse = causal_attn_fwd(c.q, c.k.cuda(), c.v.cuda(), c.cu.cpu().numpy(), c.scale, cu_seqlens_k=c.cu_k)
        # each is within 2^-8 (P |V| + |out|) of the definition; P |V| <= max |V|, whose largest of normals is below 6
        assert (got.double() - ref.double()).abs().max() <= 2 * 1.25 * 2.0 ** -8 * (6.0 + ref.abs().max().item())
        # each within 2^-20 and D 2^-24 scale |q| |k|, the latter about 128 x 0.088 x 110 x 2^-24 = 2^-13.7 here
        assert (lse - ref_lse).abs().max() <= 2.0 ** -12
        err = (got.double() - ref.double()).norm() / ref.double().norm()
        log(f"  {H}/{Hk}x{D}: {err:.2e} of the norm apart")
        assert err <= 2 * 2.0 ** -8


def test_streams_threads_and_determinism():
    import threading
    log("case streams")
    cases = [Case(12, 4, 128, 32, [1] * 9, [50 + 300 * i for i in range(9)]), Case(6, 2, 64, 16, [1, 200], [900, 400])]
    refs = [paged_attn_fwd(c.q, c.pages, c.cu, c.scale) for c in cases]
    torch.cuda.synchronize()
    bad = []

    def work(i):
        stream = torch.cuda.Stream()
        for _ in range(20):
            got = paged_attn_fwd(cases[i].q, cases[i].pages, cases[i].cu, cases[i].scale, stream=stream)
            stream.synchronize()
            if not all(torch.equal(a, b) for a, b in zip(got, refs[i])):
                bad.append(i)

    threads = [threading.Thread(target=work, args=(i % 2,)) for i in range(4)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert not bad


def test_captured_calls_follow_lengths_and_tables():
    """One graph of a step; lengths grow, a table changes and a sequence ends between its replays."""
    log("case capture")
    keys = [100, 63, 300, 16]
    c = Case(12, 4, 128, 16, [1] * 4, [n + 40 for n in keys])
    c.pages.lengths.copy_(torch.tensor(keys))
    paged_attn_fwd(c.q, c.pages, c.cu, c.scale)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for _ in range(2):  # two graphs that share a memory pool, and so workspaces
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, pool=graphs[0].pool() if graphs else None):
            outs.append(paged_attn_fwd(c.q, c.pages, c.cu, c.scale))
        graphs.append(graph)
    for i in range(30):
        c.pages.lengths.add_(1)
        c.q.mul_(-1.01)
        if i == 10:
            c.pages.table[1, :2] = c.pages.table[1, :2].flip(0).clone()
        if i == 20:
            c.pages.lengths[0] = 0
        graphs[i % 2].replay()
        eager = paged_attn_fwd(c.q, c.pages, c.cu, c.scale)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs[i % 2], eager)), i


def test_the_checked_library_agrees_and_its_checks_see(monkeypatch):
    log("case checked")
    c = Case(6, 2, 128, 16, [1, 40, 1], [100, 60, 33])
    ref = paged_attn_fwd(c.q, c.pages, c.cu, c.scale)
    with use_checked_library():
        got = paged_attn_fwd(c.q, c.pages, c.cu, c.scale)
        assert all(torch.equal(a, b) for a, b in zip(got, ref))
        monkeypatch.setenv("T2V_CHECK_CANARY", "1")
        with pytest.raises(RuntimeError, match="paged forward"):
            paged_attn_fwd(c.q, c.pages, c.cu, c.scale)
