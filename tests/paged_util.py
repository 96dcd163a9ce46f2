"""A paged cache made from packed keys and values, for tests: pages in random order, NaN in every place that holds no key, and
table entries behind a sequence's last page that no cache has."""
import numpy as np
import torch

from paper_2607_01701_amd import Pages


class Case:
    """queries, keys: tokens of each sequence. q, k, v: packed; pages: the cache that holds k and v."""

    def __init__(self, H, Hk, D, page, queries, keys, seed=0, heads_first=False, fused=False, extra_rows=0, width=None, scale=None,
                 spare=3, device="cuda"):
        g = torch.Generator().manual_seed(seed + sum(queries) + sum(keys))
        mk = lambda *s: torch.randn(s, generator=g).bfloat16()  # noqa: E731
        self.H, self.Hk, self.D, self.page, self.queries, self.keys = H, Hk, D, page, queries, keys
        self.T, Tk = sum(queries) + extra_rows, sum(keys)
        self.scale = D ** -0.5 if scale is None else scale
        self.q = mk(self.T, H + Hk if fused else H, D)[:, :H].to(device)
        self.k, self.v = mk(Tk, Hk, D), mk(Tk, Hk, D)
        self.cu = torch.tensor(np.concatenate([[0], np.cumsum(queries)]), dtype=torch.int32, device=device)
        self.cu_k = np.concatenate([[0], np.cumsum(keys)]).astype(np.int32)
        counts = [-(-n // page) for n in keys]
        n_pages = sum(counts) + spare
        order = torch.randperm(n_pages, generator=g).to(torch.int32)
        width = max([1, *counts]) + 1 if width is None else width
        table = torch.full((len(keys), width), 2 ** 31 - 1, dtype=torch.int32)
        table[:, 1::2] = -7
        shape = (n_pages, Hk, page, D) if heads_first else (n_pages, page, Hk, D)
        kp, vp = (torch.full(shape, float("nan"), dtype=torch.bfloat16) for _ in range(2))
        if heads_first:
            kp, vp = kp.transpose(1, 2), vp.transpose(1, 2)
        at = 0
        self.slots = []  # page and row of every key
        for s, n in enumerate(keys):
            table[s, :counts[s]] = order[at:at + counts[s]]
            at += counts[s]
            j = torch.arange(n)
            self.slots.append((table[s][j // page].long(), j % page))
        where = tuple(torch.cat(x) if x else torch.zeros(0, dtype=torch.long) for x in zip(*self.slots)) if keys else ()
        if Tk:
            kp[where], vp[where] = self.k, self.v
        self.where = where
        lengths = torch.tensor(keys, dtype=torch.int32)
        self.pages = Pages(kp.to(device), vp.to(device), table.to(device), lengths.to(device))
