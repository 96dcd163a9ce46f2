"""Attention over a paged cache, storing tokens and norms on the GPU where single calls go wrong: weights of many keys that cancel, odd values that
every query sees, several tokens to a workgroup, calls beyond the caches, deep sums and heads of any size."""
import numpy as np
import pytest
import torch

from oracle import norm_rotary as oracle
from paper_2607_01701_amd import Pages, norm_rotary, norm_rotary_apply, norm_rotary_bwd, paged_append, paged_attn_fwd, rotary_frequencies

from gpu_util import log
from paged_util import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def np64(x):
    return None if x is None else x.detach().double().cpu().numpy()


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("H,D,keys", [(8, 128, [64, 320, 32]), (8, 64, [320, 128]), (3, 128, [96])])
def test_single_tokens_weights_have_more_than_16_bits(H, D, keys, page):
    """The last key's value takes all others' weighted sum away, so that out is small beside its terms and an error of the weights P shows."""
    log(f"case weights {H}x{D} {keys} page {page}")
    c = Case(H, H, D, page, [1] * len(keys), keys)
    c.q.mul_(0.125)  # weights of one size
    q, k = np64(c.q), np64(c.k)
    for s, n in enumerate(keys):  # a head's weights, and the last value
        a, b = c.cu_k[s], c.cu_k[s + 1]
        x = np.einsum("hd,nhd->hn", q[s], k[a:b]) * c.scale
        p = np.exp(x - x.max(1, keepdims=True))
        p /= p.sum(1, keepdims=True)
        v = np64(c.v[a:b])
        last = -np.einsum("hn,nhd->hd", p[:, :-1], v[:-1]) / p[:, -1:]
        c.v[b - 1] = torch.from_numpy(last).bfloat16()
        pages, rows = c.slots[s]
        c.pages.v[pages[-1], rows[-1]] = c.v[b - 1].cuda()
        v[-1] = np64(c.v[b - 1])
        ref, size = np.einsum("hn,nhd->hd", p, v), np.einsum("hn,nhd->hd", p, np.abs(v))
        out, _ = paged_attn_fwd(c.q, c.pages, c.cu, c.scale)
        # P in two bf16 parts: 2^-8 of the 2^-8 that the first leaves. Scores: sums of D terms, twice (a weight and the sum of all); exp in 32 bits: 2^-20; sums over
        # the keys: n roundings of their magnitudes; out itself: 2^-8.
        score = D * 2.0 ** -24 * c.scale * np.einsum("hd,nhd->hn", np.abs(q[s]), np.abs(k[a:b])).max()
        bound = (2.0 ** -16 + 2 * score + 2.0 ** -20 + n * 2.0 ** -24) * size + 2.0 ** -8 * np.abs(ref)
        worst = float((np.abs(np64(out[s]) - ref) / bound).max())
        log(f"  {n} keys: {worst:.3f} of the bound")
        assert worst <= 1.0


@pytest.mark.parametrize("D", [64, 128])
def test_infinities_that_a_token_sees(D):
    """An infinite value gives that infinity, also at the key with the largest weight, whose rounding leaves nothing."""
    log(f"case infinities {D}")
    c = Case(4, 2, D, 16, [1, 1], [320, 64])
    p, r = c.slots[0]
    clean, clean_lse = paged_attn_fwd(c.q, c.pages, c.cu, c.scale)
    x = np.einsum("gd,nd->gn", np64(c.q)[0, :2], np64(c.k)[:320, 0])
    for j in (int(x[0].argmax()), int(x[0].argmin()), 100, 319):
        for value in (float("inf"), -float("inf")):
            old = c.pages.v[p[j], r[j], 0, 5].clone()
            c.pages.v[p[j], r[j], 0, 5] = value
            out, lse = paged_attn_fwd(c.q, c.pages, c.cu, c.scale)
            assert (out[0, :2, 5] == value).all() and torch.equal(lse, clean_lse)
            same = torch.ones_like(out, dtype=torch.bool)
            same[0, :2, 5] = False
            assert torch.equal(out[same], clean[same])
            c.pages.v[p[j], r[j], 0, 5] = old
    c.pages.v[p[7], r[7], 1, 3] = float("nan")
    out, _ = paged_attn_fwd(c.q, c.pages, c.cu, c.scale)
    assert out[0, 2:, 3].isnan().all() and int(out.isnan().sum()) == 2


@pytest.mark.parametrize("H,Hk,D,queries,keys", [(24, 8, 128, [300], [2000]), (12, 4, 64, [200, 1, 40], [900, 1500, 40]), (8, 2, 128, [1, 1], [3000, 33])])
def test_idle_sequences_change_nothing(H, Hk, D, queries, keys):
    """A cache's other sequences, without queries, some with keys: the same bits as without them."""
    log(f"case idle {H}/{Hk}x{D} {queries} over {keys}")
    c = Case(H, Hk, D, 64, queries, keys)
    ref = paged_attn_fwd(c.q, c.pages, c.cu, c.scale)
    for n in (64, 256):
        at = np.sort(np.random.default_rng(n).permutation(n)[:len(queries)])
        table = torch.full((n, c.pages.table.shape[1]), -1, dtype=torch.int32, device="cuda")
        lengths = torch.zeros(n, dtype=torch.int32, device="cuda")
        lengths[::3] = 5
        table[at], lengths[at] = c.pages.table, c.pages.lengths
        cu = torch.from_numpy(np.concatenate([[0], np.cumsum(np.bincount(at, queries, n))]).astype(np.int32)).cuda()
        got = paged_attn_fwd(c.q, Pages(c.pages.k, c.pages.v, table, lengths), cu, c.scale)
        assert all(torch.equal(a, b) for a, b in zip(got, ref))


def within(got, ref, bound, what):
    e = np.abs(np64(got) - ref)
    worst = float((e / (bound + 1e-300)).max()) if e.size else 0.0
    log(f"  {what}: {worst:.3f} of the bound")
    assert worst <= 1.0, what


@pytest.mark.parametrize("layout,pairs,D", [("half", 32, 64), ("interleaved", 40, 128), ("half", 21, 128)])
@pytest.mark.parametrize("eps,powers", [(0.0, [0, -40, -50, -70, -74, -80, -100, -115]), (1e-6, [0, 40, 58, 62, 66, 100, 120]), (1e-30, [-60, -45, -75]),
                                        (0.0, [63, 100]), (1e37, [0, 70])])
def test_heads_of_any_size(eps, powers, layout, pairs, D):
    """Heads whose squares pass the range of 32 bits either way are normalised like all others, and so are their gradients."""
    log(f"case sizes {eps} {powers} {layout} {pairs} of {D}")
    g = torch.Generator().manual_seed(len(powers) + D)
    T = len(powers) * 3
    size = torch.tensor(powers, dtype=torch.float64).repeat(3)[:, None, None]
    q, k = ((torch.randn(T, h, D, generator=g, dtype=torch.float64).clamp(-4, 4) * 2.0 ** size).bfloat16().cuda() for h in (5, 2))
    dq, dk = (torch.randn(T, h, D, generator=g).bfloat16().cuda() for h in (5, 2))
    w = (1.0 + 0.25 * torch.randn(D, generator=g)).cuda()
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    freqs, _ = rotary_frequencies(pairs)
    turn = (pos.cpu().numpy(), freqs, layout, (pairs,), 1.0)
    y = norm_rotary_apply(q, k, pos, freqs, w, w, eps, layout)
    d = norm_rotary_bwd(q, k, dq, dk, pos, freqs, w, w, eps, layout)
    n = torch.arange(T, dtype=torch.int64)
    pages = Pages(*(torch.zeros(T, 16, 2, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)),
                  n[None].int().cuda(), torch.tensor([T], dtype=torch.int32, device="cuda"))
    qa = paged_append(k, k, pages, torch.tensor([0, T], dtype=torch.int32, device="cuda"), q=q, positions=pos, freqs=freqs, layout=layout, q_weight=w,
                      k_weight=w, eps=eps)
    assert torch.equal(qa, y[0]) and torch.equal(pages.k[n // 16, n % 16], y[1])
    # A result below the smallest normal number, 2^-126, is rounded by up to 2^-134 whatever its size.
    for x, o, dy, dx, dw in ((q, y[0], dq, d[0], d[2]), (k, y[1], dk, d[1], d[3])):
        ref, bound = oracle.forward(np64(x), np64(w), float(np.float32(eps)), *turn)
        within(o, ref, bound + 2.0 ** -134, "normalised")
        ref, ref_w, bound, bound_w = oracle.backward(np64(x), np64(dy), np64(w), float(np.float32(eps)), *turn, weight_step=2.0 ** -24)
        within(dx, ref, bound + 2.0 ** -134, "gradient")
        within(dw, ref_w, bound_w, "weight's gradient")


def test_smallest_numbers_and_heads_of_one():
    """Heads of the smallest numbers of the type, and heads with one element that is not zero; a head of zeros and no eps is 0 / 0."""
    log("case smallest")
    x = torch.zeros(4, 1, 128, dtype=torch.bfloat16, device="cuda")
    x.view(torch.int16)[0] = 1  # 2^-133
    x.view(torch.int16)[1, 0, 5] = 1
    x[2, 0, 7] = -3.0e38
    y, _ = norm_rotary_apply(x, None, None, None, eps=0.0)
    assert (y[0] == 1.0).all()
    root = torch.tensor(128.0 ** 0.5).bfloat16().item()
    assert y[1, 0, 5] == root and int((y[1] != 0).sum()) == 1 and y[2, 0, 7] == -root and int((y[2] != 0).sum()) == 1
    assert y[3].isnan().all()


def test_a_chunk_leaves_tokens_their_workspace():
    """A call takes the workspace of calls of its size, whatever larger ones the same pages had before."""
    log("case workspace")
    def took(c, q, cu):
        torch.cuda.synchronize()
        torch.cuda.reset_peak_memory_stats()
        before = torch.cuda.memory_allocated()
        paged_attn_fwd(q, c.pages, cu, c.scale)
        return torch.cuda.max_memory_allocated() - before

    c = Case(12, 4, 128, 64, [2000], [4000], width=1000)
    one = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    token = [took(c, c.q[:1], one) for _ in range(2)]
    chunk = [took(c, c.q, c.cu) for _ in range(2)]
    again = [took(c, c.q[:1], one), took(c, c.q, c.cu), took(c, c.q[:10], torch.tensor([0, 10], dtype=torch.int32, device="cuda"))]
    log(f"  {token} {chunk} {again}")
    assert chunk[1] > 2 * token[1] and again[0] == token[1] and again[1] == chunk[1] and again[2] < chunk[1] / 2
