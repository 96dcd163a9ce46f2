"""A paged cache of keys and values with the attention that reads it, and the norms in front of it, as measured cases.

A causal video or caption model that answers many requests at once keeps their keys and values in pages of a
few tokens each, which a table on the GPU assigns to sequences: answers grow, fork and end without moving each other.
Each layer normalises the heads of its queries and keys, turns them by their positions, stores keys and values, and
attends; in training the norm and the turn run forward and backward.

Queries, keys and values are bf16, [tokens, heads, head_dim]; pages are [pages, page_size, kv_heads, head_dim].
Sequence s has its queries in rows cu_seqlens[s] .. cu_seqlens[s + 1] - 1 and lengths[s] keys, those of its queries the
last; its query i of Lq sees keys 0 .. i + lengths[s] - Lq. Key j is row j % page_size of page table[s, j // page_size].

With ``own`` false ``run`` computes the operators from elementary operations in 32 bits; with it true it
makes the package's calls.
"""
import math

import numpy as np
import torch

own = False

# Latent grids (as in the package's workloads) and the tokens that they have.
GRIDS = {1280: "5x16x16", 6912: "9x24x32", 20280: "13x30x52"}
HETERO = [6912, 1280, 1280, 20280, 6912, 1280, 6912, 20280, 6912, 6912, 1280, 6912, 1280, 20280, 6912, 1280]
# Keys of 32 answers that are being written.
ANSWERS = [20280, 1280, 911, 6912, 4097, 333, 12001, 77, 2051, 20280, 6001, 1024, 640, 8191, 15000, 129,
           4096, 1999, 17003, 256, 6912, 9999, 31, 2500, 1280, 11111, 5003, 384, 20280, 700, 3500, 14000]
EPS = 1e-6


def _text(lengths):
    return ",".join(map(str, lengths))


def _attention(name, heads, kv_heads, head_dim, page, queries, keys, heads_first=False):
    return {"name": name, "op": "attention", "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "page": page,
            "queries": _text(queries), "keys": _text(keys), "heads_first": heads_first}


def _append(name, heads, kv_heads, head_dim, page, queries, keys, rot_dim, layout, norm=True):
    return {"name": name, "op": "append", "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "page": page,
            "queries": _text(queries), "keys": _text(keys), "rot_dim": rot_dim, "layout": layout, "norm": norm}


def _norm(name, mode, heads, kv_heads, head_dim, rot_dim, layout, shapes, weights="bf16", fused=False):
    return {"name": name, "op": "norm", "mode": mode, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim,
            "rot_dim": rot_dim, "layout": layout, "shapes": _text(shapes), "weights": weights, "fused": fused}


def _copy(name, buffers, pages, copies, page, kv_heads, head_dim):
    return {"name": name, "op": "copy", "buffers": buffers, "pages": pages, "copies": copies, "page": page,
            "kv_heads": kv_heads, "head_dim": head_dim}


def listed():
    return [
        # One token for one short answer, 30 heads of 64 over 10, pages of 16: latency counts.
        _attention("paged_token", 30, 10, 64, 16, [1], [1280]),
        # One token more for each of 32 answers, 40 heads over 8.
        _attention("paged_tokens", 40, 8, 128, 64, [1] * 32, ANSWERS),
        # Three answers extended by a chunk (the next frames), 12 heads over 4.
        _attention("paged_chunks", 12, 4, 128, 128, [768, 257, 512], [20280, 4097, 9999]),
        # A batch as it is served: 30 answers one token further while two prompts run in chunks, 24 heads over 8; each
        # head's keys of a page together.
        _attention("paged_mixed", 24, 8, 128, 32, [1] * 30 + [512, 300], ANSWERS[:30] + [4608, 300], heads_first=True),
        # What stands before each of those: the tokens' heads normalised, turned and stored.
        _append("append_tokens", 40, 8, 128, 64, [1] * 32, ANSWERS, 128, "half"),
        # A long prompt and a chunk stored, 24 heads over 8.
        _append("append_prompt", 24, 8, 128, 64, [20280, 257], [20280, 4097], 128, "half"),
        # Training on the heterogeneous batch's patches, three axes, 24 heads, interleaved pairs.
        _norm("norm_grid_train", "train", 24, 24, 128, 128, "interleaved", [GRIDS[n] for n in HETERO]),
        # Odd lengths at 30 heads of 64, 36 of 64 dimensions turned, weights in 32 bits, training.
        _norm("norm_ragged_train", "train", 30, 10, 64, 36, "half", [4097, 333, 1280, 77, 6001, 2051, 911], weights="fp32"),
        # A long prompt, read from the fused projection's output.
        _norm("norm_prompt", "infer", 24, 8, 128, 128, "half", [20280], fused=True),
        # Five forked answers: the page that each goes on writing, in the caches of 20 layers.
        _copy("fork_pages", 40, 300, 5, 16, 8, 128),
        # Pages moved together after many answers have ended, 4 layers.
        _copy("compact_pages", 8, 1500, 700, 64, 8, 128),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: any operator and head shape, lengths spread over their range, at most the cost of the largest
    listed case of its operator."""
    largest = {}
    for c in listed():
        w = work(c)
        largest[c["op"]] = max(largest.get(c["op"], 0), w["bytes"] + w["flops"] / 250)
    while True:
        heads, kv_heads, dim = rng.choice([(2, 1, 64), (30, 10, 64), (30, 30, 64), (16, 1, 64), (12, 12, 128), (12, 4, 128),
                                           (24, 8, 128), (6, 2, 128), (40, 8, 128), (3, 1, 128), (24, 24, 128)])
        op = rng.choice(["attention", "attention", "attention", "append", "norm", "norm", "copy"])
        page = rng.choice([16, 32, 64, 128, 256])
        rot = rng.choice([dim, dim, dim // 2, 2 * rng.randint(1, dim // 2)])
        layout = rng.choice(["half", "interleaved"])
        n = _log_int(rng, 1, 32)
        longest = _log_int(rng, 16, 20280)
        keys = [min(longest, _log_int(rng, max(1, longest // 64), longest * 2)) for _ in range(n)]
        tokens = [min(k, rng.choice([1, 1, 1, 2, 4])) for k in keys]
        chunks = [min(k, _log_int(rng, 4, 1024)) for k in keys]
        queries = rng.choice([tokens, tokens, chunks, [c if rng.random() < 0.1 else t for c, t in zip(chunks, tokens)]])
        if op == "attention":
            case = _attention("drawn", heads, kv_heads, dim, page, queries, keys, heads_first=rng.random() < 0.3)
            if len([q for q in queries if q > 4]) * max(queries) * heads * max(keys) > 2 ** 30:  # of the plain form's scores
                continue
        elif op == "append":
            queries = rng.choice([tokens, chunks, keys])
            case = _append("drawn", heads, kv_heads, dim, page, queries, keys, rot, layout, norm=rng.random() < 0.8)
        elif op == "norm":
            shapes = ["%dx%dx%d" % (rng.randint(1, 21), rng.randint(4, 45), rng.randint(4, 80))
                      for _ in range(_log_int(rng, 1, 12))] if rng.random() < 0.3 else rng.choice([keys, [1] * n])
            mode = rng.choice(["train", "train", "infer"])
            case = _norm("drawn", mode, heads, kv_heads, dim, dim if "x" in str(shapes[0]) else rot, layout, shapes,
                         weights=rng.choice(["bf16", "fp32", "none"]), fused=mode == "infer" and rng.random() < 0.5)
        else:
            pages = _log_int(rng, 2, 2000)
            case = _copy("drawn", _log_int(rng, 1, 48), pages, _log_int(rng, 1, pages // 2), page, kv_heads, dim)
            if case["buffers"] * pages * page * kv_heads * dim > 2 ** 30:
                continue
        w = work(case)
        if w["bytes"] + w["flops"] / 250 > largest[op]:
            continue
        del case["name"]
        return case


def _ints(text):
    return [int(x) for x in text.split(",")]


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(torch.bfloat16)


def _cu(lengths):
    return torch.from_numpy(np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)).cuda()


def _cache(case, g, keys):
    """k and v pages, the table and the lengths: pages handed out in random order, 1 in 8 free, -1 behind each sequence."""
    page, hk, d = case["page"], case["kv_heads"], case["head_dim"]
    counts = [(n + page - 1) // page for n in keys]
    n_pages = sum(counts) + sum(counts) // 8 + 1
    k, v = (_normal(g, n_pages, hk, page, d).transpose(1, 2) if case.get("heads_first") else _normal(g, n_pages, page, hk, d)
            for _ in range(2))
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    first = np.concatenate([[0], np.cumsum(counts)[:-1]])[:, None] + np.arange(max(counts))
    held = np.arange(max(counts)) < np.array(counts)[:, None]
    place = torch.from_numpy(np.where(held, first, 0)).cuda()
    table = torch.where(torch.from_numpy(held).cuda(), order[place], -1).contiguous()
    return k, v, table, torch.tensor(keys, dtype=torch.int32, device="cuda")


def _sections(case):
    """Pairs of dimensions that each axis turns."""
    pairs = case["rot_dim"] // 2
    if "x" not in case.get("shapes", ""):
        return (pairs,)
    t = pairs // 4
    return (t, (pairs - t) // 2, pairs - t - (pairs - t) // 2)


def _frequencies(case):
    """Radians a position, float64 [rot_dim / 2]."""
    return np.concatenate([10000.0 ** -(np.arange(n, dtype=np.float64) / max(n, 1)) for n in _sections(case)])


def _positions(case):
    """int32 [axes, tokens]: a token's place in its sequence, or its patch's frame, row and column."""
    if case["op"] == "append":
        return np.concatenate([np.arange(k - q, k, dtype=np.int32)
                               for q, k in zip(_ints(case["queries"]), _ints(case["keys"]))])[None]
    shapes = [[int(x) for x in s.split("x")] for s in case["shapes"].split(",")]
    if len(shapes[0]) == 3:
        return np.concatenate([np.indices(s, dtype=np.int32).reshape(3, -1) for s in shapes], axis=1)
    return np.concatenate([np.arange(s[0], dtype=np.int32) for s in shapes])[None]


def _weights(case, g):
    """Norm weights of queries and keys near one, as training leaves them."""
    if case.get("weights") == "none" or not case.get("norm", True):
        return None, None
    w = 1.0 + 0.2 * torch.randn((2, case["head_dim"]), generator=g, device="cuda")
    return tuple(w if case.get("weights") == "fp32" else w.to(torch.bfloat16))


def _inputs(case, seed):
    """The case's tensors, from the seed alone."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    st = dict(case)
    h, hk, d = case.get("heads"), case["kv_heads"], case["head_dim"]
    if case["op"] == "copy":
        st["caches"] = [_normal(g, case["pages"], case["page"], hk, d) for _ in range(case["buffers"])]
        order = torch.randperm(case["pages"], generator=g, device="cuda").cpu().numpy().astype(np.int32)
        st["src"], st["dst"] = order[:case["copies"]], order[case["copies"]:2 * case["copies"]]
        return st
    if case["op"] != "norm":
        queries, keys = _ints(case["queries"]), _ints(case["keys"])
        st["k_pages"], st["v_pages"], st["table"], st["lengths"] = _cache(case, g, keys)
        st["cu"], st["t"] = _cu(queries), sum(queries)
    if case["op"] == "attention":
        st["q"], st["scale"] = _normal(g, st["t"], h, d), 1.0 / math.sqrt(d)
        return st
    st["positions"] = torch.from_numpy(_positions(case)).cuda()
    t = st["t"] = st["positions"].shape[1]
    # Projections' outputs: their size differs from token to token.
    size = torch.exp(0.5 * torch.randn((t, 1, 1), generator=g, device="cuda"))
    if case["op"] == "append" or case["fused"]:
        qkv = torch.randn((t, h + 2 * hk, d), generator=g, device="cuda").mul_(size).to(torch.bfloat16)
        st["q"], st["k"], st["v"] = qkv[:, :h], qkv[:, h:h + hk], qkv[:, h + hk:]
    else:
        st["q"], st["k"] = (torch.randn((t, n, d), generator=g, device="cuda").mul_(size).to(torch.bfloat16) for n in (h, hk))
    if case.get("mode") == "train":
        st["dq"], st["dk"] = _normal(g, t, h, d), _normal(g, t, hk, d)
    st["wq"], st["wk"] = _weights(case, g)
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    if case["op"] in ("append", "norm"):
        st["freqs"], st["sections"] = _frequencies(case), _sections(case)
        if not own:
            st["freqs"] = torch.from_numpy(st["freqs"]).cuda()
    if own and case["op"] in ("append", "attention"):
        from paper_2607_01701_amd import Pages
        st["pages"] = Pages(st["k_pages"], st["v_pages"], st["table"], st["lengths"])
    if own and case.get("mode") == "train":
        for n in ("q", "k", "wq", "wk"):
            if st[n] is not None:
                st[n].requires_grad_(True)
    return st


# ------------------------------------------------------------------------ plain forms


def _normed(x, w):
    """x in 32 bits times its reciprocal root mean square, that, and the result times the weights."""
    x = x.float()
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    return x * r, r, x * r if w is None else x * r * w.float()


def _turned(y, cos, sin, layout, rot):
    a, b = (y[..., 0:rot:2], y[..., 1:rot:2]) if layout == "interleaved" else (y[..., :rot // 2], y[..., rot // 2:rot])
    c, d = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack((c, d), -1).flatten(-2) if layout == "interleaved" else torch.cat((c, d), -1)
    return torch.cat((turned, y[..., rot:]), -1)


def _angles(st):
    """Cosines and sines [tokens, 1, pairs]; the angles in 64 bits."""
    axis = torch.repeat_interleave(torch.arange(len(st["sections"])), torch.tensor(st["sections"])).cuda()
    angle = (st["positions"][axis].t().double() * st["freqs"])[:, None]
    return torch.cos(angle).float(), torch.sin(angle).float()


def _plain_norm(st):
    cos, sin = _angles(st)
    layout, rot = st["layout"], st["rot_dim"]
    out, dx, dw = [], [], []
    for x, w, dy in ((st["q"], st["wq"], st.get("dq")), (st["k"], st["wk"], st.get("dk"))):
        xhat, r, n = _normed(x, w)
        out.append(_turned(n, cos, sin, layout, rot).to(torch.bfloat16))
        if st["mode"] == "train":
            dn = _turned(dy.float(), cos, -sin, layout, rot)
            g = dn if w is None else dn * w.float()
            dx.append((r * (g - xhat * (g * xhat).mean(-1, keepdim=True))).to(torch.bfloat16))
            if w is not None:
                dw.append((dn * xhat).sum((0, 1)).to(w.dtype))
    return (*out, *dx, *dw)


def _slots(st):
    """Page and row of each new token."""
    queries = st["cu"][1:] - st["cu"][:-1]
    seq = torch.repeat_interleave(torch.arange(len(queries), device="cuda"), queries, output_size=st["t"])
    place = torch.arange(st["t"], device="cuda") - st["cu"][seq] + (st["lengths"] - queries)[seq]
    return st["table"][seq, place // st["page"]].long(), place % st["page"]


def _plain_append(st):
    cos, sin = _angles(st)
    q, k = ((_normed(x, w)[2] if st["norm"] else x.float()) for x, w in ((st["q"], st["wq"]), (st["k"], st["wk"])))
    at = _slots(st)
    st["k_pages"][at] = _turned(k, cos, sin, st["layout"], st["rot_dim"]).to(torch.bfloat16)
    st["v_pages"][at] = st["v"]
    return _turned(q, cos, sin, st["layout"], st["rot_dim"]).to(torch.bfloat16), st["k_pages"], st["v_pages"]


def _attend(st, seqs, out, lse):
    """The sequences `seqs` (a list), padded to the longest of them."""
    queries, keys = np.array(_ints(st["queries"]))[seqs], np.array(_ints(st["keys"]))[seqs]
    h, hk, d, n = st["heads"], st["kv_heads"], st["head_dim"], len(seqs)
    lq, lk, g = int(queries.max()), int(keys.max()), st["heads"] // st["kv_heads"]
    at = torch.tensor(seqs, device="cuda")
    count, length = (st["cu"][1:] - st["cu"][:-1])[at], st["lengths"][at]
    j = torch.arange(lk, device="cuda")
    page = st["table"][at][:, j // st["page"]].clamp(min=0).long()
    k, v = (x[page, j % st["page"]].float().transpose(1, 2).contiguous() for x in (st["k_pages"], st["v_pages"]))
    i = torch.arange(lq, device="cuda")
    row = (st["cu"][at][:, None] + torch.minimum(i, count[:, None] - 1)).long()
    q = st["q"][row].float().view(n, lq, hk, g, d).permute(0, 2, 1, 3, 4).reshape(n, hk, lq * g, d)
    x = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(st["scale"])
    last = (i + (length - count)[:, None]).repeat_interleave(g, 1)[:, None, :, None]
    x.masked_fill_(j > last, -math.inf)
    m = x.amax(3, keepdim=True)
    x.sub_(torch.where(m == -math.inf, 0.0, m)).exp_()
    s = x.sum(3, keepdim=True)
    o = torch.matmul(x, v).div_(torch.where(s == 0.0, 1.0, s))
    real = i < count[:, None]
    out[row[real]] = o.view(n, hk, lq, g, d).permute(0, 2, 1, 3, 4).reshape(n, lq, h, d)[real].to(torch.bfloat16)
    lse[:, row[real]] = (m + torch.log(s)).view(n, hk, lq, g).permute(0, 2, 1, 3).reshape(n, lq, h)[real].t()


def _plain_attention(st):
    out = torch.empty_like(st["q"])
    lse = torch.empty((st["heads"], st["t"]), dtype=torch.float32, device="cuda")
    queries = _ints(st["queries"])
    few, many = [s for s, n in enumerate(queries) if n <= 4], [s for s, n in enumerate(queries) if n > 4]
    if few:
        _attend(st, few, out, lse)
    if many:
        _attend(st, many, out, lse)
    return out, lse


def _plain_copy(st):
    src, dst = (torch.from_numpy(x.astype(np.int64)).cuda() for x in (st["src"], st["dst"]))
    for cache in st["caches"]:
        cache[dst] = cache[src]
    return st["caches"]


def run(st):
    if not own:
        return {"attention": _plain_attention, "append": _plain_append, "norm": _plain_norm, "copy": _plain_copy}[st["op"]](st)
    import paper_2607_01701_amd as t2v
    if st["op"] == "copy":
        t2v.page_copy(st["caches"], st["src"], st["dst"])
        return st["caches"]
    if st["op"] == "attention":
        return t2v.paged_attn_fwd(st["q"], st["pages"], st["cu"], st["scale"])
    if st["op"] == "append":
        q = t2v.paged_append(st["k"], st["v"], st["pages"], st["cu"], q=st["q"], positions=st["positions"], freqs=st["freqs"],
                             layout=st["layout"], sections=st["sections"], q_weight=st["wq"], k_weight=st["wk"],
                             eps=EPS if st["norm"] else None)
        return q, st["k_pages"], st["v_pages"]
    q, k = t2v.norm_rotary(st["q"], st["k"], st["positions"], st["freqs"], q_weight=st["wq"], k_weight=st["wk"], eps=EPS,
                           layout=st["layout"], sections=st["sections"])
    if st["mode"] == "infer":
        return q, k
    leaves = [st[n] for n in ("q", "k", "wq", "wk") if st[n] is not None]
    return (q.detach(), k.detach(), *torch.autograd.grad((q, k), leaves, (st["dq"], st["dk"])))


def work(case):
    """Inputs read once and outputs written once. Attention: two products of every visible pair, 2 flops per multiply-add.
    Norms: an element takes three flops for its square and two products, a pair six for its turn; twice that
    backward. Stored tokens count with their pages' rows, not the pages that stay as they are."""
    h, hk, d = case.get("heads", 0), case["kv_heads"], case["head_dim"]
    if case["op"] == "copy":
        return {"bytes": 2 * case["buffers"] * case["copies"] * case["page"] * hk * d * 2, "flops": 0}
    if case["op"] == "norm":
        t = sum(math.prod(int(x) for x in s.split("x")) for s in case["shapes"].split(","))
        train = case["mode"] == "train"
        return {"bytes": (10 if train else 4) * t * (h + hk) * d + 4 * t * len(_sections(case)),
                "flops": (3 if train else 1) * t * (h + hk) * (3 * d + 3 * case["rot_dim"])}
    queries, keys = _ints(case["queries"]), _ints(case["keys"])
    t, page = sum(queries), case["page"]
    if case["op"] == "append":
        return {"bytes": 4 * t * (h + 2 * hk) * d + 4 * t, "flops": t * (h + hk) * (3 * d + 3 * case["rot_dim"])}
    pairs = sum(k * q - q * (q - 1) // 2 for q, k in zip(queries, keys))
    return {"bytes": 4 * t * h * d + 4 * t * h + 4 * sum(keys) * hk * d + 4 * sum(-(-k // page) for k in keys),
            "flops": 4 * h * d * pairs}


# --------------------------------------------------------------- the definitions in 64 bits


def exact(case, seed):
    return {"attention": _exact_attention, "append": _exact_append, "norm": _exact_norm, "copy": _exact_copy}[case["op"]](
        case, _inputs(case, seed))


def _exact_attention(case, st):
    queries, keys, page = _ints(case["queries"]), _ints(case["keys"]), case["page"]
    group, t = case["heads"] // case["kv_heads"], st["t"]
    out = torch.zeros((t, case["heads"], case["head_dim"]), dtype=torch.float64, device="cuda")
    lse = torch.zeros((case["heads"], t), dtype=torch.float64, device="cuda")
    table, row = st["table"].cpu().numpy(), 0
    for s, (n, m) in enumerate(zip(queries, keys)):
        pages = torch.from_numpy(table[s, :(m + page - 1) // page].astype(np.int64)).cuda()
        sees = torch.arange(m, device="cuda")[None] <= torch.arange(m - n, m, device="cuda")[:, None]
        for j in range(case["kv_heads"]):
            k, v = (x[pages, :, j].reshape(-1, case["head_dim"])[:m].double() for x in (st["k_pages"], st["v_pages"]))
            for h in range(j * group, (j + 1) * group):
                score = st["q"][row:row + n, h].double() @ k.t() / math.sqrt(case["head_dim"])
                score = torch.where(sees, score, -math.inf)
                lse[h, row:row + n] = torch.logsumexp(score, 1)
                out[row:row + n, h] = torch.softmax(score, 1) @ v
        row += n
    return out, lse


def _rotations(case):
    """exp(i angle) of each token and pair."""
    axis = np.repeat(np.arange(len(_sections(case))), _sections(case))
    return torch.exp(1j * torch.from_numpy(_positions(case)[axis].T * _frequencies(case)).cuda())[:, None]


def _exact_turn(y, z, case):
    """The pairs of y, as complex numbers, times z."""
    rot = case["rot_dim"]
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if case["layout"] == "interleaved" else (slice(0, rot // 2), slice(rot // 2, rot))
    z = torch.complex(y[..., a], y[..., b]) * z
    y = y.clone()
    y[..., a], y[..., b] = z.real, z.imag
    return y


def _exact_norm(case, st):
    z = _rotations(case)
    out, dx, dw = [], [], []
    for x, w, dy in ((st["q"], st["wq"], st.get("dq")), (st["k"], st["wk"], st.get("dk"))):
        x, weight = x.double(), 1.0 if w is None else w.double()
        size = ((x ** 2).sum(-1, keepdim=True) / x.shape[-1] + EPS) ** 0.5
        out.append(_exact_turn(x / size * weight, z, case))
        if case["mode"] == "train":
            dn = _exact_turn(dy.double(), z.conj(), case)
            # d(x / size) = dx / size - x (x . dx) / (D size^3)
            back = dn * weight
            dx.append(back / size - x * (back * x).sum(-1, keepdim=True) / (x.shape[-1] * size ** 3))
            if w is not None:
                dw.append(torch.einsum("thd,thd->d", dn, x / size))
    return (*out, *dx, *dw)


def _exact_append(case, st):
    z = _rotations(case)
    turned = []
    for x, w in ((st["q"], st["wq"]), (st["k"], st["wk"])):
        x = x.double()
        if case["norm"]:
            x = x / ((x ** 2).sum(-1, keepdim=True) / x.shape[-1] + EPS) ** 0.5 * (1.0 if w is None else w.double())
        turned.append(_exact_turn(x, z, case))
    k_pages, v_pages = st["k_pages"].double(), st["v_pages"].double()
    table, row, page = st["table"].cpu().numpy(), 0, case["page"]
    for s, (n, m) in enumerate(zip(_ints(case["queries"]), _ints(case["keys"]))):
        place = np.arange(m - n, m)
        at = tuple(torch.from_numpy(x.astype(np.int64)).cuda() for x in (table[s, place // page], place % page))
        k_pages[at], v_pages[at] = turned[1][row:row + n], st["v"][row:row + n].double()
        row += n
    return turned[0], k_pages, v_pages


def _exact_copy(case, st):
    of = np.arange(case["pages"])
    of[st["dst"]] = st["src"]
    of = torch.from_numpy(of).cuda()
    return [cache.index_select(0, of).double() for cache in st["caches"]]
