"""Causal attention with grouped heads and rotary positions, as measured cases.

A causal video or caption model trains on packed sequences of different lengths, and answers by
running a prompt, extending it by a chunk, or adding single tokens to long caches of keys and
values. Its queries have more heads than its keys and values; heads are turned by their positions
(one axis for text, frame / height / width for latent patches) before the attention.

Queries, keys and values are bf16, packed token-major [tokens, heads, head_dim]; query i of a
sequence with Lq queries and Lk keys sees keys 0 .. i + Lk - Lq. Values are N(0, 1), the softmax
scale is 1 / sqrt(head_dim).

With ``own`` false ``run`` computes the operators from elementary products and sums in 32 bits;
with it true it makes the package's calls.
"""
import math

import numpy as np
import torch

own = False

# Latent grids and what they are (as in the package's workloads).
IMAGE = 1 * 32 * 32          # 1,024 tokens
SHORT_CLIP = 5 * 16 * 16     # 1,280
MID_CLIP = 9 * 24 * 32       # 6,912
LONG_CLIP = 13 * 30 * 52     # 20,280
HETERO = [MID_CLIP, SHORT_CLIP, SHORT_CLIP, LONG_CLIP, MID_CLIP, SHORT_CLIP, MID_CLIP, LONG_CLIP,
          MID_CLIP, MID_CLIP, SHORT_CLIP, MID_CLIP, SHORT_CLIP, LONG_CLIP, MID_CLIP, SHORT_CLIP]
GRIDS = {SHORT_CLIP: "5x16x16", MID_CLIP: "9x24x32", LONG_CLIP: "13x30x52"}
# Keys already in the caches of 32 answers that are being written.
CACHES = [20280, 1280, 911, 6912, 4097, 333, 12001, 77, 2051, 20280, 6001, 1024, 640, 8191, 15000, 129,
          4096, 1999, 17003, 256, 6912, 9999, 31, 2500, 1280, 11111, 5003, 384, 20280, 700, 3500, 14000]


def _attention(name, mode, heads, kv_heads, head_dim, lengths, lengths_k=None, fused=False):
    return {"name": name, "op": "attention", "mode": mode, "heads": heads, "kv_heads": kv_heads,
            "head_dim": head_dim, "lengths": ",".join(map(str, lengths)),
            "lengths_k": ",".join(map(str, lengths if lengths_k is None else lengths_k)), "fused": fused}


def _rotary(name, mode, heads, kv_heads, head_dim, rot_dim, layout, shapes, scaling="none", start=0, fused=False):
    return {"name": name, "op": "rotary", "mode": mode, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim,
            "rot_dim": rot_dim, "layout": layout, "shapes": ",".join(map(str, shapes)), "scaling": scaling,
            "start": start, "fused": fused}


def listed():
    return [
        # The smallest training step: two captions at 2 heads of 64; launches and host work count.
        _attention("tiny_train", "train", 2, 1, 64, [256, 384]),
        # Captions and clips cropped to odd sizes, 30 heads of 64 over 10.
        _attention("ragged_d64_train", "train", 30, 10, 64, [4097, 333, 1280, 77, 6001, 2051, 911]),
        # Equal clips of 4,096 tokens, 24 heads of 128 over 8.
        _attention("uniform_train", "train", 24, 8, 128, [4096] * 8),
        # The heterogeneous batch, every one of 12 heads with keys of its own.
        _attention("hetero_train", "train", 12, 12, 128, HETERO),
        # Running one long prompt, 24 heads over 8, read from the fused projection's output.
        _attention("long_prompt", "infer", 24, 8, 128, [LONG_CLIP], fused=True),
        # Extending three answers by a chunk (the next frames) over what is cached, 12 heads over 4.
        _attention("chunk_over_cache", "infer", 12, 4, 128, [768, 257, 512], [20280, 4097, 9999]),
        # One token more for each of 32 answers, 40 heads over 8.
        _attention("tokens_batch", "infer", 40, 8, 128, [1] * len(CACHES), CACHES),
        # One token for one short answer, 30 heads of 64 over 10: latency counts.
        _attention("token_single", "infer", 30, 10, 64, [1], [1280]),
        # The heterogeneous batch's patches, three axes, training: 24 heads, interleaved pairs.
        _rotary("grid_train", "train", 24, 24, 128, 128, "interleaved", [GRIDS[n] for n in HETERO]),
        # Odd lengths at 30 heads of 64, half layout, 36 of 64 dimensions turned, training.
        _rotary("ragged_partial_train", "train", 30, 10, 64, 36, "half", [4097, 333, 1280, 77, 6001, 2051, 911]),
        # A long prompt beyond the trained context, read from the fused projection: wavelengths scaled by ramp.
        _rotary("scaled_prompt", "infer", 24, 8, 128, 64, "half", [LONG_CLIP], scaling="yarn", fused=True),
        # 32 single tokens at far positions, 40 heads over 8: latency counts.
        _rotary("far_tokens", "infer", 40, 8, 128, 128, "half", [1] * 32, start=1_000_003),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: any operator, direction and head shape, lengths spread over their range, at
    most the cost of the largest listed case of its operator."""
    by = {c["name"]: c for c in listed()}
    most = work(by["uniform_train"])["flops"]
    most_bytes = work(by["grid_train"])["bytes"]
    while True:
        heads, kv_heads, dim = rng.choice([(2, 1, 64), (2, 2, 64), (30, 10, 64), (30, 30, 64), (15, 5, 64),
                                           (16, 1, 64), (12, 12, 128), (12, 4, 128), (24, 8, 128), (6, 2, 128),
                                           (40, 8, 128), (10, 2, 128), (3, 1, 128), (24, 24, 128)])
        kind = rng.choice(["train", "train", "prompt", "chunk", "token", "rotary", "rotary"])
        n = _log_int(rng, 1, 32)
        longest = _log_int(rng, 64, LONG_CLIP)
        lengths = [min(longest, _log_int(rng, max(1, longest // 32), longest * 2)) for _ in range(n)]
        if kind == "rotary":
            axes = rng.choice([1, 1, 3])
            if axes == 3:
                shapes = ["%dx%dx%d" % (rng.randint(1, 21), rng.randint(4, 45), rng.randint(4, 80))
                          for _ in range(_log_int(rng, 1, 12))]
                rot = dim
            else:
                shapes = [1] * n if rng.random() < 0.3 else lengths
                rot = rng.choice([dim, dim, dim // 2, 2 * rng.randint(1, dim // 2)])
            case = _rotary("drawn", rng.choice(["train", "infer"]), heads, kv_heads, dim, rot,
                           rng.choice(["half", "interleaved"]), shapes,
                           rng.choice(["none", "linear", "ntk", "yarn"]) if axes == 1 else "none",
                           rng.choice([0, rng.randint(1, 2_000_000)]) if axes == 1 else 0)
            case["fused"] = case["mode"] == "infer" and rng.random() < 0.5
            if work(case)["bytes"] > most_bytes:
                continue
        else:
            if kind == "token":
                lq, lk = [rng.choice([1, 1, 1, 2, 4])] * n, [x + 4 for x in lengths]
            elif kind == "chunk":
                lk = lengths
                lq = [min(k, _log_int(rng, 8, 1024)) for k in lk]
            else:
                lq = lk = lengths
            case = _attention("drawn", "train" if kind == "train" else "infer", heads, kv_heads, dim, lq, lk,
                              fused=kind == "prompt" and rng.random() < 0.5)
            if work(case)["flops"] > most or sum(lk) * heads * dim > 2 ** 29:
                continue
        del case["name"]
        return case


def _ints(text):
    return [int(x) for x in text.split(",")]


def _cu(lengths):
    return np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(torch.bfloat16)


def _attention_inputs(case, seed):
    """q, k, v, dout; with ``fused`` q, k and v are slices of one projection's output."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    h, hk, d = case["heads"], case["kv_heads"], case["head_dim"]
    tq, tk = sum(_ints(case["lengths"])), sum(_ints(case["lengths_k"]))
    if case["fused"]:
        qkv = _normal(g, tq, h + 2 * hk, d)
        return qkv[:, :h], qkv[:, h:h + hk], qkv[:, h + hk:], None
    q, k, v = _normal(g, tq, h, d), _normal(g, tk, hk, d), _normal(g, tk, hk, d)
    return q, k, v, _normal(g, tq, h, d) if case["mode"] == "train" else None


def _tokens(case):
    return sum(math.prod(int(x) for x in s.split("x")) for s in case["shapes"].split(","))


def _positions(case):
    """int32 [axes, tokens]: a token's place in its sequence, or its patch's frame, row and column."""
    shapes = [[int(x) for x in s.split("x")] for s in case["shapes"].split(",")]
    if len(shapes[0]) == 3:
        return np.concatenate([np.indices(s, dtype=np.int32).reshape(3, -1) for s in shapes], axis=1)
    return np.concatenate([np.arange(s[0], dtype=np.int32) + case["start"] for s in shapes])[None]


def _sections(case):
    """Pairs of dimensions that each axis turns."""
    pairs = case["rot_dim"] // 2
    if "x" not in case["shapes"]:
        return (pairs,)
    t = pairs // 4
    return (t, (pairs - t) // 2, pairs - t - (pairs - t) // 2)


TRAINED, FACTOR = 4096, 8.0  # of the scaled frequencies: positions trained on, and how much further they reach


def _frequencies(case):
    """Radians a position, float64 [rot_dim / 2], and the factor on the turned dimensions."""
    freqs = []
    for n in _sections(case):
        j = np.arange(n, dtype=np.float64) / n
        theta = 10000.0
        if case["scaling"] == "ntk" and n > 1:
            theta *= FACTOR ** (n / (n - 1))
        f = theta ** -j
        if case["scaling"] == "linear":
            f = f / FACTOR
        elif case["scaling"] == "yarn":
            keep = np.clip((TRAINED * f / (2 * np.pi) - 1.0) / (32.0 - 1.0), 0.0, 1.0)
            f = f * keep + f / FACTOR * (1.0 - keep)
        freqs.append(f)
    return np.concatenate(freqs), 0.1 * math.log(FACTOR) + 1.0 if case["scaling"] == "yarn" else 1.0


def _rotary_inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    h, hk, d, t = case["heads"], case["kv_heads"], case["head_dim"], _tokens(case)
    if case["fused"]:
        qkv = _normal(g, t, h + 2 * hk, d)
        return qkv[:, :h], qkv[:, h:h + hk], None, None
    q, k = _normal(g, t, h, d), _normal(g, t, hk, d)
    return (q, k, _normal(g, t, h, d), _normal(g, t, hk, d)) if case["mode"] == "train" else (q, k, None, None)


def prepare(case, seed):
    st = {"op": case["op"], "mode": case["mode"]}
    if case["op"] == "attention":
        st["q"], st["k"], st["v"], st["dout"] = _attention_inputs(case, seed)
        st["cu"], st["scale"] = _cu(_ints(case["lengths"])), 1.0 / math.sqrt(case["head_dim"])
        st["cu_k"] = None if case["lengths"] == case["lengths_k"] else _cu(_ints(case["lengths_k"]))
        leaves = ("q", "k", "v")
    else:
        st["q"], st["k"], st["dq"], st["dk"] = _rotary_inputs(case, seed)
        st["positions"] = torch.from_numpy(_positions(case)).cuda()
        st["layout"], st["sections"], st["rot"] = case["layout"], _sections(case), case["rot_dim"]
        if own:
            from paper_2607_01701_amd import rotary_frequencies
            scaling = None if case["scaling"] == "none" else case["scaling"]
            st["freqs"], st["mscale"] = rotary_frequencies(st["sections"], 10000.0, scaling=scaling, factor=FACTOR,
                                                           trained=TRAINED)
        else:
            freqs, st["mscale"] = _frequencies(case)
            st["freqs"] = torch.from_numpy(freqs).cuda()
        leaves = ("q", "k")
    if own and case["mode"] == "train":
        for n in leaves:
            st[n].requires_grad_(True)
    return st


# ------------------------------------------------------------------------ plain forms


def _plain_attention(st):
    q, k, v, dout, scale = st["q"], st["k"], st["v"], st["dout"], st["scale"]
    cu, cu_k = st["cu"].tolist(), (st["cu"] if st["cu_k"] is None else st["cu_k"]).tolist()
    (tq, h, d), hk = q.shape, k.shape[1]
    g = h // hk
    out = torch.zeros((tq, h, d), dtype=torch.bfloat16, device=q.device)
    lse = torch.full((h, tq), -math.inf, dtype=torch.float32, device=q.device)
    train = dout is not None
    if train:
        dq, dk, dv = (torch.zeros_like(x) for x in (q, k, v))

    def grouped(x, a, b):  # rows a .. b of [T, H, D] as [Hk, (b - a) g, D] in 32 bits
        return x[a:b].float().view(b - a, hk, g, d).permute(1, 0, 2, 3).reshape(hk, (b - a) * g, d)

    def packed(x, n):  # and back
        return x.view(hk, n, g, d).permute(1, 0, 2, 3).reshape(n, h, d)

    for s in range(len(cu) - 1):
        lq, lk = cu[s + 1] - cu[s], cu_k[s + 1] - cu_k[s]
        if lq == 0 or lk == 0:
            continue
        kk = k[cu_k[s]:cu_k[s + 1]].float().permute(1, 0, 2).contiguous()
        vv = v[cu_k[s]:cu_k[s + 1]].float().permute(1, 0, 2).contiguous()
        kt, vt = kk.transpose(1, 2).contiguous(), vv.transpose(1, 2).contiguous()
        if train:
            dks, dvs = torch.zeros_like(kk), torch.zeros_like(vv)
        step = max(1, (1 << 27) // (h * lk))
        for a in range(0, lq, step):
            b = min(a + step, lq)
            n = b + lk - lq  # keys that the chunk's last query sees
            if n <= 0:
                continue
            rows = slice(cu[s] + a, cu[s] + b)
            qq = grouped(q, cu[s] + a, cu[s] + b)
            x = torch.matmul(qq, kt[:, :, :n].contiguous()) * scale
            last = torch.arange(a, b, device=q.device).repeat_interleave(g) + (lk - lq)
            x.masked_fill_(torch.arange(n, device=q.device) > last[:, None], -math.inf)
            m = x.amax(2, keepdim=True)
            x = torch.exp(x - torch.where(m == -math.inf, 0.0, m))
            l = x.sum(2, keepdim=True)
            x = x / torch.where(l == 0.0, 1.0, l)
            o = torch.matmul(x, vv[:, :n])
            out[rows] = packed(o, b - a).to(torch.bfloat16)
            lse[:, rows] = (m + torch.log(l)).view(hk, b - a, g).permute(0, 2, 1).reshape(h, b - a)
            if train:
                go = grouped(dout, cu[s] + a, cu[s] + b)
                dvs[:, :n] += torch.matmul(x.transpose(1, 2).contiguous(), go)
                dp = torch.matmul(go, vt[:, :, :n].contiguous())
                x = x * (dp - (go * o).sum(2, keepdim=True)) * scale
                dks[:, :n] += torch.matmul(x.transpose(1, 2).contiguous(), qq)
                dq[rows] = packed(torch.matmul(x, kk[:, :n]), b - a).to(torch.bfloat16)
        if train:
            dk[cu_k[s]:cu_k[s + 1]] = dks.permute(1, 0, 2).to(torch.bfloat16)
            dv[cu_k[s]:cu_k[s + 1]] = dvs.permute(1, 0, 2).to(torch.bfloat16)
    return (out, lse, dq, dk, dv) if train else (out, lse)


def _turn(x, cos, sin, layout, rot):
    y = x.float()
    a, b = (y[..., 0:rot:2], y[..., 1:rot:2]) if layout == "interleaved" else (y[..., :rot // 2], y[..., rot // 2:rot])
    c, d = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack((c, d), -1).flatten(-2) if layout == "interleaved" else torch.cat((c, d), -1)
    return torch.cat((turned, y[..., rot:]), -1).to(torch.bfloat16)


def _plain_rotary(st):
    # Angles in 64 bits: a far position times its frequency needs more than 24 bits.
    parts = torch.split(st["freqs"], list(st["sections"]))
    angle = torch.cat([p[:, None].double() * f for p, f in zip(st["positions"], parts)], 1)[:, None]
    cos, sin = (torch.cos(angle) * st["mscale"]).float(), (torch.sin(angle) * st["mscale"]).float()
    back = (st["dq"], st["dk"]) if st["mode"] == "train" else ()
    return tuple(_turn(x, cos, sin, st["layout"], st["rot"]) for x in (st["q"], st["k"])) + tuple(
        _turn(x, cos, -sin, st["layout"], st["rot"]) for x in back)


def run(st):
    if not own:
        return _plain_attention(st) if st["op"] == "attention" else _plain_rotary(st)
    import paper_2607_01701_amd as t2v
    if st["op"] == "attention":
        if st["mode"] == "infer":
            return t2v.causal_attn_fwd(st["q"], st["k"], st["v"], st["cu"], st["scale"], cu_seqlens_k=st["cu_k"])
        out, lse = t2v.varlen_causal_attention(st["q"], st["k"], st["v"], st["cu"], st["scale"],
                                               cu_seqlens_k=st["cu_k"])
        return (out.detach(), lse, *torch.autograd.grad(out, (st["q"], st["k"], st["v"]), st["dout"]))
    q, k = t2v.rotary(st["q"], st["k"], st["positions"], st["freqs"], layout=st["layout"], sections=st["sections"],
                      mscale=st["mscale"])
    if st["mode"] == "infer":
        return q, k
    return (q.detach(), k.detach(), *torch.autograd.grad((q, k), (st["q"], st["k"]), (st["dq"], st["dk"])))


def work(case):
    """Inputs read once and outputs written once. Attention: two products of every visible pair
    forward and five backward, 2 flops per multiply-add. Rotary: a product of a pair of dimensions
    with a 2 x 2 matrix is six flops."""
    h, hk, d = case["heads"], case["kv_heads"], case["head_dim"]
    passes = 2 if case["mode"] == "train" else 1
    if case["op"] == "rotary":
        t = _tokens(case)
        axes = 3 if "x" in case["shapes"] else 1
        return {"bytes": passes * 4 * t * (h + hk) * d + 4 * t * axes,
                "flops": passes * 3 * t * (h + hk) * case["rot_dim"]}
    lq, lk = _ints(case["lengths"]), _ints(case["lengths_k"])
    pairs = sum(b * a - a * (a - 1) // 2 if a <= b else b * (b + 1) // 2 for a, b in zip(lq, lk))
    tq, tk = sum(lq), sum(lk)
    # q, k, v in, out and lse out; training: dout in, dq, dk, dv out.
    moved = 2 * d * (2 * tq * h + 2 * tk * hk) + 4 * tq * h
    if case["mode"] == "train":
        moved += 2 * d * (2 * tq * h + 2 * tk * hk)
    return {"bytes": moved, "flops": (7 if case["mode"] == "train" else 2) * 2 * h * d * pairs}


# --------------------------------------------------------------- the definitions in 64 bits


def exact(case, seed):
    if case["op"] == "rotary":
        return _exact_rotary(case, seed)
    # Loops over heads and sequences that are many would take too long, and so would the largest products.
    lq, lk = _ints(case["lengths"]), _ints(case["lengths_k"])
    if work(case)["flops"] > 4e13 or len(lq) * case["heads"] > 4000:
        return None
    q, k, v, dout = _attention_inputs(case, seed)
    cu, cu_k, scale = _cu(lq).tolist(), _cu(lk).tolist(), 1.0 / math.sqrt(case["head_dim"])
    group = case["heads"] // case["kv_heads"]
    train = dout is not None
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.full((q.shape[1], q.shape[0]), -math.inf, dtype=torch.float64, device="cuda")
    if train:
        dq, dk, dv = (torch.zeros(x.shape, dtype=torch.float64, device="cuda") for x in (q, k, v))
    for s in range(len(lq)):
        if lk[s] == 0:
            continue
        for h in range(case["heads"]):
            j = h // group
            kh, vh = k[cu_k[s]:cu_k[s + 1], j].double(), v[cu_k[s]:cu_k[s + 1], j].double()
            step = max(1, (1 << 26) // lk[s])
            for a in range(0, lq[s], step):
                b = min(a + step, lq[s])
                r = slice(cu[s] + a, cu[s] + b)
                sees = torch.arange(lk[s], device="cuda")[None] <= torch.arange(a, b, device="cuda")[:, None] + (
                    lk[s] - lq[s])
                qh = q[r, h].double()
                score = torch.where(sees, qh @ kh.t() * scale, -math.inf)
                norm = torch.logsumexp(score, 1)
                prob = torch.where(sees, torch.exp(score - norm[:, None]), 0.0)
                o = prob @ vh
                out[r, h], lse[h, r] = o, norm
                if train:
                    go = dout[r, h].double()
                    grad = prob * (go @ vh.t() - (go * o).sum(1, keepdim=True)) * scale
                    dq[r, h] = grad @ kh
                    dk[cu_k[s]:cu_k[s + 1], j] += grad.t() @ qh
                    dv[cu_k[s]:cu_k[s + 1], j] += prob.t() @ go
    return (out, lse, dq, dk, dv) if train else (out, lse)


def _exact_rotary(case, seed):
    """Pairs as complex numbers times exp(i angle), a sequence of the same positions at a time."""
    q, k, dq, dk = _rotary_inputs(case, seed)
    freqs, mscale = _frequencies(case)
    axis = np.repeat(np.arange(len(_sections(case))), _sections(case))
    angle = torch.from_numpy(_positions(case)[axis].T.astype(np.float64) * freqs).cuda()
    rot = case["rot_dim"]

    def turned(x, sign):
        y = x.double()
        first, second = (slice(0, rot, 2), slice(1, rot, 2)) if case["layout"] == "interleaved" else (
            slice(0, rot // 2), slice(rot // 2, rot))
        z = torch.complex(y[..., first], y[..., second]) * (mscale * torch.exp(1j * sign * angle))[:, None]
        y[..., first], y[..., second] = z.real, z.imag
        return y

    forward = (turned(q, 1), turned(k, 1))
    return forward if case["mode"] != "train" else (*forward, turned(dq, -1), turned(dk, -1))
