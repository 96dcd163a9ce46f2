"""Storing new tokens in pages and copying pages on the GPU, and all of a paged cache's calls together as a model makes them: a block
that normalises, turns, stores and attends, token by token, with forks, ends and compaction, against whole sequences."""
import numpy as np
import pytest
import torch

from oracle import causal_attention
from oracle import norm_rotary as oracle
from paper_2607_01701_amd import (PagedCache, Pages, causal_attn_fwd, norm_rotary_apply, page_copy, paged_append, paged_attn_fwd,
                                  rotary_apply, rotary_frequencies)

from gpu_util import log
from paged_util import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def bits(x):
    return x.contiguous().view(torch.int16)


def new_tokens(c):
    """Page and row of each new token of a Case, in order."""
    p = [s[0][n - q:] for s, q, n in zip(c.slots, c.queries, c.keys)]
    r = [s[1][n - q:] for s, q, n in zip(c.slots, c.queries, c.keys)]
    return torch.cat(p), torch.cat(r)


CASES = [  # H, Hk, D, page, queries, keys, pairs
    (40, 8, 128, 64, [1] * 5, [1, 64, 65, 300, 17], 64), (30, 10, 64, 16, [20, 1, 0, 40], [20, 100, 7, 55], 18),
    (3, 1, 128, 32, [33, 2], [200, 2], 21), (2, 2, 64, 256, [1], [256], 32), (12, 4, 128, 16, [700, 1, 300], [900, 33, 300], 40),
    (1, 16, 64, 16, [3] * 70, [16] * 70, 7),
]


@pytest.mark.parametrize("heads_first", [False, True], ids=["tokens", "heads"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("H,Hk,D,page,queries,keys,pairs", CASES)
def test_append(H, Hk, D, page, queries, keys, pairs, layout, heads_first):
    log(f"case append {H}/{Hk}x{D} page {page} {queries[:5]} over {keys[:5]} {pairs} {layout}")
    c = Case(H, Hk, D, page, queries, keys, heads_first=heads_first, extra_rows=3)
    g = torch.Generator().manual_seed(9)
    qkv = torch.randn(c.T, H + 2 * Hk, D, generator=g).bfloat16().cuda()
    q, k, v = qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:]
    n, at = sum(queries), new_tokens(c)
    wq, wk = ((1.0 + 0.3 * torch.randn(D, generator=g)).bfloat16().cuda() for _ in range(2))
    pos = torch.arange(c.T, dtype=torch.int32, device="cuda") * 7 - 3
    freqs, _ = rotary_frequencies(pairs)
    other = torch.ones(c.pages.k.shape[:2], dtype=torch.bool)
    other[at] = False
    forms = {"plain": {}, "norm": dict(q=q, eps=1e-6, q_weight=wq, k_weight=wk),
             "turn": dict(q=q, positions=pos, freqs=freqs, layout=layout),
             "both": dict(q=q, positions=pos, freqs=freqs, layout=layout, eps=1e-5, q_weight=wq, mscale=1.5),
             "keys": dict(positions=pos, freqs=freqs, layout=layout, eps=1e-5, k_weight=wk)}
    for name, kw in forms.items():
        c = Case(H, Hk, D, page, queries, keys, heads_first=heads_first, extra_rows=3)
        before = (bits(c.pages.k).cpu(), bits(c.pages.v).cpu())
        q_out = torch.full((c.T, H, D), 7.0, dtype=torch.bfloat16, device="cuda") if "q" in kw else None
        got = paged_append(k, v, c.pages, c.cu, q_out=q_out, **kw)
        torch.cuda.synchronize()
        assert got is q_out
        for pages, old, src in ((c.pages.k, before[0], k), (c.pages.v, before[1], v)):
            assert torch.equal(bits(pages).cpu()[other], old[other])  # the other rows stay
        assert torch.equal(bits(c.pages.v)[at], bits(v[:n]))
        if name == "plain":
            assert torch.equal(bits(c.pages.k)[at], bits(k[:n]))
            continue
        turn = (pos[:n].cpu().numpy(), freqs, layout, (pairs,), kw.get("mscale", 1.0)) if "freqs" in kw else (None,) * 5
        for x, y, w in ((q, q_out, kw.get("q_weight")), (k, c.pages.k[at], kw.get("k_weight"))):
            if y is None:
                continue
            x, w = x[:n].double().cpu().numpy(), None if w is None else w.double().cpu().numpy()
            if "eps" in kw:
                ref, bound = oracle.forward(x, w, kw["eps"], *turn)
            else:
                ref, bound = oracle.turned(x, 0.0 * x, *turn)
                bound = bound + 2.0 ** -8 * np.abs(ref)
            e = np.abs(y[:n].double().cpu().numpy() - ref)
            assert (e <= bound + 1e-300).all(), name
        if q_out is not None:
            assert (q_out[n:] == 7.0).all()


def test_append_copies_every_bit():
    """Keys and values that are stored as they are keep the bits of their infinities and NaN."""
    log("case bits")
    c = Case(2, 2, 64, 16, [20, 3], [20, 30])
    g = torch.Generator().manual_seed(3)
    k, v = (torch.randint(-2 ** 15, 2 ** 15, (c.T, 2, 64), generator=g).to(torch.int16).view(torch.bfloat16).cuda() for _ in range(2))
    paged_append(k, v, c.pages, c.cu)
    at = new_tokens(c)
    assert torch.equal(bits(c.pages.k)[at], bits(k)) and torch.equal(bits(c.pages.v)[at], bits(v))
    freqs, _ = rotary_frequencies(8)
    pos = torch.arange(c.T, dtype=torch.int32, device="cuda")
    paged_append(k, v, c.pages, c.cu, positions=pos, freqs=freqs)
    assert torch.equal(bits(c.pages.v)[at], bits(v))
    _, turned = rotary_apply(None, k, pos, freqs)
    assert torch.equal(c.pages.k[at].isnan(), turned.isnan())


def test_append_without_a_place():
    """Pages outside the cache, keys below 0 and beyond the table: not stored, and nothing else is touched."""
    log("case no place")
    c = Case(4, 2, 64, 16, [3, 2, 4], [30, 20, 40])
    k = torch.ones(c.T, 2, 64, dtype=torch.bfloat16, device="cuda")
    before = bits(c.pages.k).clone()
    c.pages.table.fill_(-1)
    paged_append(k, k.clone(), c.pages, c.cu)
    assert torch.equal(bits(c.pages.k), before)
    c.pages.table.fill_(2 ** 31 - 1)
    paged_append(k, k.clone(), c.pages, c.cu)
    assert torch.equal(bits(c.pages.k), before)
    c.pages.table.copy_(torch.arange(3)[:, None].expand_as(c.pages.table))
    room = c.pages.table.shape[1] * 16
    c.pages.lengths.copy_(torch.tensor([0, room + 1, 2]))  # no key; too long; only the last two of four have a place
    paged_append(k, k.clone(), c.pages, c.cu)
    changed = (bits(c.pages.k) != before).flatten(2).any(2).nonzero().tolist()
    assert changed == [[2, 0], [2, 1]]
    for cu in ([0, 5, 2, 9], [-5, 3, 1000, 2000], [9, 9, 9, 9], [2 ** 31 - 1, -2 ** 31, 0, 4]):
        q = torch.full((c.T + 8, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
        paged_append(k, k.clone(), c.pages, torch.tensor(cu, dtype=torch.int32, device="cuda"), q=q[:c.T].clone(), eps=1e-6, q_out=q[:c.T])
        torch.cuda.synchronize()
        assert (q[c.T:] == 7.0).all()


@pytest.mark.parametrize("shape,dtype,n", [((7, 16, 2, 64), torch.bfloat16, 3), ((1000, 16, 1, 64), torch.bfloat16, 450),
                                           ((40, 3, 5, 16), torch.float32, 20), ((9, 16), torch.uint8, 4), ((5, 64, 40, 128), torch.bfloat16, 2)])
def test_page_copy(shape, dtype, n):
    log(f"case copy {shape} {dtype} {n}")
    g = torch.Generator().manual_seed(n)
    bufs = [torch.randint(0, 255, (*shape[:-1], shape[-1] * dtype.itemsize), generator=g).to(torch.uint8).cuda().view(dtype) for _ in range(3)]
    order = torch.randperm(shape[0], generator=g).numpy()
    src, dst = np.resize(order[:max(1, n // 2)], n), order[shape[0] - n:]  # pages copied to several
    refs = [b.clone().view(torch.uint8) for b in bufs]
    for r in refs:
        r[dst] = r[src]
    page_copy(bufs, src, dst)
    assert all(torch.equal(b.view(torch.uint8), r) for b, r in zip(bufs, refs))
    page_copy(bufs[0], [], [])


def test_page_copy_of_strided_pages_and_many_buffers():
    log("case copy strided")
    whole = torch.randn(20, 75, 2, 16, 2, 64, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    ref = whole.clone()
    ref[[3, 4, 19]] = ref[[0, 1, 1]]
    page_copy([whole[:, i, j] for i in range(75) for j in range(2)], [0, 1, 1], [3, 4, 19])
    assert torch.equal(whole, ref)
    heads = torch.randn(6, 2, 16, 64).bfloat16().cuda()
    ref = heads.clone()
    ref[5] = ref[2]
    page_copy(heads.transpose(1, 2), [2], [5], stream=torch.cuda.current_stream())
    assert torch.equal(heads, ref)


def test_page_copy_of_more_than_the_caches_hold():
    log("case copy 290 MB")
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randint(-2 ** 31, 2 ** 31 - 1, (2, 1700, 32771, 4), dtype=torch.int32, device="cuda", generator=g)[:, :, :8195]  # a part's end in a page, a gap between pages
    ref = x.clone()
    ref[:, 550:1100] = ref[:, 1100:1650] = ref[:, :550]
    page_copy([x[0], x[1]], np.arange(1100) % 550, np.arange(550, 1650))
    assert torch.equal(x, ref)


def test_page_copy_beyond_32_bit_offsets():
    log("case copy large")
    x = torch.zeros(40_000, 64 * 8 * 128, dtype=torch.bfloat16, device="cuda")
    x[39_999] = 3.0
    x[1] = 2.0
    page_copy(x, [39_999, 1], [0, 39_998])
    assert (x[0] == 3.0).all() and (x[39_998] == 2.0).all() and (x[2:39_998] == 0).all()


def test_captured_append_and_copy():
    log("case captured append")
    c = Case(6, 2, 128, 16, [1, 1, 1], [40, 80, 60])
    c.pages.lengths.copy_(torch.tensor([5, 17, 30]))
    k, v, q = (torch.randn(3, h, 128).bfloat16().cuda() for h in (2, 2, 6))
    freqs, _ = rotary_frequencies(64)
    pos = torch.zeros(3, dtype=torch.int32, device="cuda")
    kw = dict(q=q, positions=pos, freqs=freqs, eps=1e-6)
    twin = Pages(c.pages.k.clone(), c.pages.v.clone(), c.pages.table, c.pages.lengths)
    free = [p for p in range(c.pages.k.shape[0]) if p not in set(torch.cat([s[0] for s in c.slots]).tolist())]
    pairs = ([int(c.slots[0][0][0])], [free[0]])
    paged_append(k, v, c.pages, c.cu, **kw)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.pages.lengths.add_(1)
        pos.copy_(c.pages.lengths)
        out = paged_append(k, v, c.pages, c.cu, **kw)
        page_copy([c.pages.k, c.pages.v], *pairs)
    paged_append(k, v, twin, c.cu, **kw)  # as the call before the capture
    for i in range(12):
        k.mul_(-1.1)
        graph.replay()
        ref = paged_append(k, v, twin, c.cu, **kw)
        page_copy([twin.k, twin.v], *pairs)
        torch.cuda.synchronize()
        assert torch.equal(out, ref) and torch.equal(bits(twin.k), bits(c.pages.k)) and torch.equal(bits(twin.v), bits(c.pages.v)), i


class Block:
    """Two layers of a small model: projections, norm, turn, attention, output projection."""

    def __init__(self, H, Hk, D, seed=0):
        g = torch.Generator().manual_seed(seed)
        mk = lambda *s: (torch.randn(s, generator=g) / s[0] ** 0.5).bfloat16().cuda()  # noqa: E731
        self.H, self.Hk, self.D, self.E = H, Hk, D, 96
        self.layers = [dict(qkv=mk(96, (H + 2 * Hk) * D), out=mk(H * D, 96), wq=(1 + 0.1 * torch.randn(D, generator=g)).cuda(),
                            wk=(1 + 0.1 * torch.randn(D, generator=g)).cuda()) for _ in range(2)]
        self.freqs, _ = rotary_frequencies(D // 2)
        self.scale = D ** -0.5

    def qkv(self, x, w):
        y = (x @ w["qkv"]).view(x.shape[0], self.H + 2 * self.Hk, self.D)
        return y[:, :self.H], y[:, self.H:self.H + self.Hk], y[:, self.H + self.Hk:]

    def whole(self, x, lengths):
        """Packed sequences at once, with the packed calls."""
        pos = torch.cat([torch.arange(n) for n in lengths]).int().cuda()
        cu = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
        for w in self.layers:
            q, k, v = self.qkv(x, w)
            q, k = norm_rotary_apply(q, k, pos, self.freqs, w["wq"], w["wk"])
            o, _ = causal_attn_fwd(q, k, v.contiguous(), cu, self.scale)
            x = x + o.view(x.shape[0], -1) @ w["out"]
        return x

    def paged(self, x, cache, cu, pos):
        for i, w in enumerate(self.layers):
            q, k, v = self.qkv(x, w)
            q = paged_append(k, v, cache.layer(i), cu, q=q, positions=pos, freqs=self.freqs, q_weight=w["wq"], k_weight=w["wk"], eps=1e-6)
            o, _ = paged_attn_fwd(q, cache.layer(i), cu, self.scale)
            x = x + o.view(x.shape[0], -1) @ w["out"]
        return x


def close(a, b):
    """Two ways of the same block: every step rounds to bf16 (2^-8) in another order of sums, in two layers of five roundings with an
    addition to the stream each; independent, they leave about 2^-8 of the norm, of which four times is allowed."""
    e = ((a.double() - b.double()).norm() / b.double().norm()).item()
    log(f"  {e:.2e} of the norm apart")
    assert e <= 4 * 2.0 ** -8


def test_a_block_over_the_cache_with_forks_ends_and_compaction():
    log("case block")
    H, Hk, D = 6, 2, 64
    block = Block(H, Hk, D)
    cache = PagedCache(2, 60, Hk, D, page_size=16, sequences=6, width=12)
    g = torch.Generator().manual_seed(4)
    text = {}  # inputs of each sequence
    token = lambda n: torch.randn(n, 96, generator=g).bfloat16().cuda()  # noqa: E731

    def step(new):
        """new: tokens of some sequences; all others have none."""
        seqs = sorted(new)
        cache.extend(seqs, [new[s].shape[0] for s in seqs])
        pos = torch.cat([torch.arange(text[s].shape[0], text[s].shape[0] + new[s].shape[0]) for s in seqs]).int().cuda()
        y = block.paged(torch.cat([new[s] for s in seqs]), cache, cache.offsets({s: new[s].shape[0] for s in seqs}), pos)
        at = 0
        for s in seqs:
            n = new[s].shape[0]
            text[s] = torch.cat([text[s], new[s]])
            close(y[at:at + n], block.whole(text[s], [text[s].shape[0]])[-n:])
            at += n

    a, b, c = cache.add(), cache.add(), cache.add()
    for s in (a, b, c):
        text[s] = token(0)
    step({a: token(37), c: token(5)})           # two prompts
    step({a: token(1), b: token(50), c: token(1)})  # a prompt among single tokens
    f = cache.fork(a)
    text[f] = text[a].clone()
    step({a: token(1), f: token(1)})            # they differ from here on
    cache.free(c)
    del text[c]
    assert cache.compact() >= 0
    step({a: token(12), b: token(1), f: token(30)})  # chunks
    cache.truncate(b, 40)
    text[b] = text[b][:40]
    cache.compact()
    used = int((cache.host.refs > 0).sum())
    assert (cache.host.refs[:used] > 0).all() and cache.free_pages == 60 - used
    step({s: token(1) for s in (a, b, f)})
    with pytest.raises(RuntimeError, match="pages"):
        cache.extend([a, b, f], [600, 600, 600])
    step({a: token(1)})
    torch.cuda.synchronize()
    assert torch.equal(cache.lengths.cpu(), torch.from_numpy(cache.host.lengths)) and torch.equal(cache.table.cpu(), torch.from_numpy(cache.host.table))


def test_a_captured_block_writes_an_answer():
    """One graph of a step for two sequences, replayed as they grow through several pages, beside eager calls on another cache."""
    log("case captured block")
    H, Hk, D = 6, 2, 128
    block = Block(H, Hk, D, seed=1)
    g = torch.Generator().manual_seed(6)
    prompts = [torch.randn(n, 96, generator=g).bfloat16().cuda() for n in (29, 3)]
    cache = PagedCache(2, 30, Hk, D, page_size=16, sequences=2, width=10)
    for p in prompts:
        s = cache.add()
        cache.extend([s], [p.shape[0]])
        block.paged(p, cache, cache.offsets({s: p.shape[0]}), torch.arange(p.shape[0], dtype=torch.int32, device="cuda"))
    cache.reserve([0, 1], 60)
    cu = cache.offsets([1, 1])
    x = torch.zeros(2, 96, dtype=torch.bfloat16, device="cuda")
    pos = torch.zeros(2, dtype=torch.int32, device="cuda")

    def step():
        pos.copy_(cache.lengths)
        cache.lengths.add_(1)
        return block.paged(x, cache, cu, pos)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        cache.lengths.sub_(1)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = step()
        with pytest.raises(RuntimeError, match="captured"):
            cache.extend([0], [1])
        with pytest.raises(RuntimeError, match="captured"):
            cache.offsets([1, 1])
    texts = list(prompts)
    for i in range(40):
        x.copy_(torch.randn(2, 96, generator=g))
        graph.replay()
        texts = [torch.cat([t, x[j:j + 1]]) for j, t in enumerate(texts)]
        if i % 8 == 7:
            for j, t in enumerate(texts):
                close(y[j:j + 1], block.whole(t, [t.shape[0]])[-1:])
    cache.grown([0, 1], 40)
    torch.cuda.synchronize()
    assert torch.equal(cache.lengths.cpu(), torch.from_numpy(cache.host.lengths))


def test_cache_offsets_and_tables_on_the_gpu():
    log("case offsets and tables")
    cache = PagedCache(1, 40, 1, 64, page_size=16, sequences=3, width=20)
    assert cache.offsets({2: 5, 0: 3}).tolist() == [0, 3, 3, 8] and cache.offsets([1, 2]).tolist() == [0, 1, 3, 3]
    for bad in ({3: 1}, {-1: 1}, {0: -1}, [1, 1, 1, 1], {0: 2 ** 31 - 1, 1: 1}):
        with pytest.raises(ValueError, match="tokens"):
            cache.offsets(bad)
    r = np.random.default_rng(2)
    a, b = cache.add(), cache.add()
    for step in range(40):  # longer, shorter, none
        s = (a, b)[step % 2]
        do = r.integers(0, 3)
        if do == 0:
            cache.truncate(s, int(r.integers(0, cache.host.lengths[s] + 1)))
        elif do == 1 and cache.host.lengths[s] < 200:
            cache.extend([s], [int(r.integers(0, 90))])
        else:
            cache.compact()
        assert torch.equal(cache.table.cpu(), torch.from_numpy(cache.host.table))
        assert torch.equal(cache.lengths.cpu(), torch.from_numpy(cache.host.lengths))


def test_the_definition_end_to_end():
    """Append and attention together against the float64 definitions, with the stored keys' own rounding in between."""
    log("case end to end")
    H, Hk, D, queries, keys = 6, 2, 64, [4, 20], [60, 20]
    c = Case(H, Hk, D, 16, queries, keys)
    freqs, _ = rotary_frequencies(32)
    q, k, v = (torch.randn(24, h, D, generator=torch.Generator().manual_seed(h)).bfloat16().cuda() for h in (H, Hk, Hk + 1))
    v = v[:, :Hk]
    pos = torch.cat([torch.arange(56, 60), torch.arange(20)]).int().cuda()
    qn = paged_append(k, v, c.pages, c.cu, q=q, positions=pos, freqs=freqs, eps=1e-6)
    out, lse = paged_attn_fwd(qn, c.pages, c.cu, c.scale)
    kk, vv = (x[c.where].double().cpu().numpy() for x in (c.pages.k, c.pages.v))
    ref = causal_attention(qn.double().cpu().numpy(), kk, vv, None, np.array([0, 4, 24]), c.cu_k, c.scale)
    assert (np.abs(out.double().cpu().numpy() - ref["out"]) <= ref["bounds"]["out"]).all()
    assert (np.abs(lse.double().cpu().numpy() - ref["lse"]) <= ref["bounds"]["lse"]).all()
    n, bound = oracle.forward(k.double().cpu().numpy(), None, 1e-6, pos.cpu().numpy(), freqs, "half", (32,), 1.0)
    assert (np.abs(c.pages.k[new_tokens(c)].double().cpu().numpy() - n) <= bound).all()
