"""Attention over a paged cache, storing tokens and norms on the GPU where single calls go wrong: weights of many keys that cancel, odd values that
every query sees, several tokens to a workgroup, calls beyond the caches, deep sums and heads of any size."""
import numpy as np
import pytest
import torch

from paper_2607_01701_amd import Pages, paged_attn_fwd

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
