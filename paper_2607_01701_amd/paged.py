"""Paged caches of keys and values (t2v_pages): the description that the calls take, attention over them, and what fills and moves
their pages. The binding marshals arguments; the computation is in the HIP library."""
from __future__ import annotations

import ctypes

from . import _lib


class Pages:
    """The pages of one layer's keys and values and the table that assigns them to sequences, as the calls take them.

    k, v: bf16 [pages, page_size, Hk, D] on the GPU, page_size a power of two from 16 on; any strides with D innermost and a page's rows
    apart (a cache [pages, Hk, page_size, D] is passed as its transpose(1, 2)). table: int32 [nseq, width] on the GPU, rows any distance
    apart: key j of sequence s is row j % page_size of page table[s, j // page_size]. lengths: int32 [nseq] on the GPU: keys of each
    sequence, those of a call's own tokens the last. The object keeps the tensors, whose contents may change between calls and between replays of a
    captured call; it is made once and passed to every call."""

    def __init__(self, k, v, table, lengths):
        import torch
        if k.dim() != 4:
            raise ValueError("k must be [pages, page_size, kv_heads, head_dim]")
        for t, name in ((k, "k"), (v, "v")):
            if t.shape != k.shape:
                raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(k.shape)}")
            if t.dtype != torch.bfloat16:
                raise ValueError(f"{name} has dtype {t.dtype}, expected {torch.bfloat16}")
            if t.stride(3) != 1:
                raise ValueError(f"{name} must hold each head contiguously, got strides {t.stride()}")
        if table.dim() != 2 or table.dtype != torch.int32 or (table.shape[1] > 1 and table.stride(1) != 1):
            raise ValueError("table must be int32 [nseq, width] with contiguous rows")
        if lengths.shape != (table.shape[0],) or lengths.dtype != torch.int32 or not lengths.is_contiguous():
            raise ValueError(f"lengths must be contiguous int32 [{table.shape[0]}]")
        _lib._check_on_device((("k", k), ("v", v), ("table", table), ("lengths", lengths)))
        self.k, self.v, self.table, self.lengths = k, v, table, lengths
        self.device = k.device
        (pages, page_size, kv_heads, head_dim), i64 = k.shape, ctypes.c_int64 * 3
        self.nseq, self.kv_heads, self.head_dim = table.shape[0], kv_heads, head_dim
        self._struct = _lib.PagesStruct(k.data_ptr(), v.data_ptr(), i64(*k.stride()[:3]), i64(*v.stride()[:3]), pages,
                                        table.data_ptr(), table.stride(0) if table.shape[0] > 1 else table.shape[1],
                                        table.shape[1], lengths.data_ptr(), table.shape[0], page_size, kv_heads, head_dim)
        self._ref = ctypes.byref(self._struct)
        self._workspace = _lib._WORKSPACE  # what the last call needed


def _check_cu(cu, pages):
    import torch
    if cu.shape != (pages.nseq + 1,) or cu.dtype != torch.int32 or not cu.is_contiguous():
        raise ValueError(f"cu_seqlens must be contiguous int32 [{pages.nseq + 1}] on the GPU")


def paged_attn_fwd(q, pages: Pages, cu_seqlens, scale: float, max_queries=None, out=None, lse=None, stream=None):
    """Causal attention with grouped heads over a paged cache: single tokens, chunks and prompts in one call. q [T, H, D] (bf16 on
    the GPU, tokens any distance apart) holds sequence s's queries in rows cu_seqlens[s] .. cu_seqlens[s + 1] - 1 (int32 on the GPU; rows behind
    the last are padding and left as they are in out and lse). Query i of Lq sees keys 0 .. i + lengths[s] - Lq of its sequence, whose
    keys and values are already stored. max_queries: the most queries of a sequence, if known (for speed). Returns (out [T, H, D]
    bf16, lse [H, T] fp32). A page number outside the cache or a length beyond the table's width gives NaN."""
    import torch
    if q.dim() != 3:
        raise ValueError("q must be [tokens, heads, head_dim]")
    T, H, D = q.shape
    if D != pages.head_dim:
        raise ValueError(f"q has head_dim {D}, the pages {pages.head_dim}")
    step = _lib._check_rows(q, "q", (T, H, D))
    _check_cu(cu_seqlens, pages)
    named = [("k", pages.k), ("q", q), ("cu_seqlens", cu_seqlens)]
    (out, lse), given = _lib._outputs((("out", out, (T, H, D), torch.bfloat16), ("lse", lse, (H, T), torch.float32)), q.device, stream)
    _lib._check_on_device((*named, *given))
    L, need = _lib.lib(), ctypes.c_uint64()
    for _ in range(2):
        size = pages._workspace
        with _lib._on(stream):
            ws = torch.empty(size, dtype=torch.uint8, device=q.device)
        st = _lib._call_on(q.device, stream, L.t2v_paged_fwd, q.data_ptr(), step, H, cu_seqlens.data_ptr(), T, max_queries or 0,
                           pages._ref, scale, out.data_ptr(), lse.data_ptr(), ws.data_ptr(), size, ctypes.byref(need))
        if st != _lib.T2V_ERR_WORKSPACE:
            break
        pages._workspace = need.value
    if st != _lib.T2V_OK:
        _lib._check(L, st)
    return out, lse
