"""Paged caches of keys and values (t2v_pages): the description that the calls take, attention over them, and what fills and moves
their pages. The binding marshals arguments; the computation is in the HIP library."""
from __future__ import annotations

import ctypes

import numpy as np

from . import _lib
from .norm_rotary import _aligned_weight, _checked, _turn_struct


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
        self._workspace = {}  # what calls needed, by the power of two that their packed rows reach


def _check_cu(cu, pages):
    import torch
    if cu.shape != (pages.nseq + 1,) or cu.dtype != torch.int32 or not cu.is_contiguous():
        raise ValueError(f"cu_seqlens must be contiguous int32 [{pages.nseq + 1}] on the GPU")


def _same_device(device, *named):
    for name, t in named:
        if t.device != device:
            if not t.is_cuda:
                raise ValueError(f"{name} must be a CUDA tensor")
            raise ValueError(f"{name} is on {t.device}, the pages on {device}")


def paged_attn_fwd(q, pages: Pages, cu_seqlens, scale: float, out=None, lse=None, stream=None):
    """Causal attention with grouped heads over a paged cache: single tokens, chunks and prompts in one call. q [T, H, D] (bf16 on
    the GPU, tokens any distance apart) holds sequence s's queries in rows cu_seqlens[s] .. cu_seqlens[s + 1] - 1 (int32 on the GPU; rows behind
    the last are padding and left as they are in out and lse). Query i of Lq sees keys 0 .. i + lengths[s] - Lq of its sequence, whose
    keys and values are already stored. Returns (out [T, H, D]
    bf16, lse [H, T] fp32). A page number outside the cache or a length beyond the table's width gives NaN. No autograd: the results have no gradient or
    tangent, whatever the arguments have."""
    import torch
    if q.dim() != 3:
        raise ValueError("q must be [tokens, heads, head_dim]")
    T, H, D = q.shape
    if D != pages.head_dim:
        raise ValueError(f"q has head_dim {D}, the pages {pages.head_dim}")
    step = _lib._check_rows(q, "q", (T, H, D))
    _check_cu(cu_seqlens, pages)
    device = pages.device
    _same_device(device, ("q", q), ("cu_seqlens", cu_seqlens))
    rows = (T * H // pages.kv_heads - 1).bit_length()
    size = pages._workspace.get(rows, _lib._WORKSPACE)
    if out is None and lse is None and stream is None:
        out = torch.empty((T, H, D), dtype=torch.bfloat16, device=device)
        lse = torch.empty((H, T), dtype=torch.float32, device=device)
        ws = torch.empty(size, dtype=torch.uint8, device=device)
    else:
        (out, lse), given = _lib._outputs((("out", out, (T, H, D), torch.bfloat16), ("lse", lse, (H, T), torch.float32)), device, stream)
        _same_device(device, *given)
        with _lib._on(stream):
            ws = torch.empty(size, dtype=torch.uint8, device=device)
    L, need = _lib.lib(), ctypes.c_uint64()
    args = (q.data_ptr(), step, H, cu_seqlens.data_ptr(), T, pages._ref, scale, out.data_ptr(), lse.data_ptr())
    st = _lib._call_on(device, stream, L.t2v_paged_fwd, *args, ws.data_ptr(), size, ctypes.byref(need))
    if st == _lib.T2V_ERR_WORKSPACE:
        size = pages._workspace[rows] = need.value  # more than any such call so far
        with _lib._on(stream):
            ws = torch.empty(size, dtype=torch.uint8, device=device)
        st = _lib._call_on(device, stream, L.t2v_paged_fwd, *args, ws.data_ptr(), size, ctypes.byref(need))
    if st != _lib.T2V_OK:
        _lib._check(L, st)
    return out, lse


def paged_append(k, v, pages: Pages, cu_seqlens, q=None, positions=None, freqs=None, layout: str = "half", sections=None,
                 mscale: float = 1.0, q_weight=None, k_weight=None, eps=None, q_out=None, stream=None):
    """Stores the keys and values k, v [T, Hk, D] of new tokens in their pages: of sequence s with Lq tokens (rows as in paged_attn_fwd), token i is key
    lengths[s] - Lq + i. With freqs and positions the keys are turned before, with eps normalised (times k_weight), and so are the
    queries q [T, H, D] of the same tokens, as by norm_rotary_apply, in the same pass; returns those (None without q). A token without a place in
    the cache is not stored, nor any of a sequence whose length passes the table's width (attention over them gives NaN). No autograd, as in paged_attn_fwd."""
    import torch
    if k.dim() != 3 or (q is not None and q.dim() != 3):
        raise ValueError("q and k must be [tokens, heads, head_dim]")
    T, D = k.shape[0], pages.head_dim
    shape = (T, pages.kv_heads, D)
    sk, sv = _lib._check_rows(k, "k", shape), _lib._check_rows(v, "v", shape)
    _check_cu(cu_seqlens, pages)
    device = pages.device
    named = [("k", k), ("v", v), ("cu_seqlens", cu_seqlens)]
    turn = None
    if freqs is not None or eps is not None:
        checked = _checked(q, k, positions, freqs, layout, sections, mscale, q_weight, k_weight, eps)
    elif q is not None or positions is not None or sections is not None or q_weight is not None or k_weight is not None:
        raise ValueError("q, positions, sections or weights are given without a norm (eps) or a turn (freqs)")
    else:
        checked = None
    sq, heads, qp, given = 0, 0, None, ()
    if q is not None:
        heads = q.shape[1]
        sq, qp = _lib._check_rows(q, "q", (T, heads, D)), q.data_ptr()
        named.append(("q", q))
        if q_out is None and stream is None:
            q_out = torch.empty((T, heads, D), dtype=torch.bfloat16, device=device)
        else:
            (q_out,), given = _lib._outputs((("q_out", q_out, (T, heads, D), torch.bfloat16),), device, stream)
    elif q_out is not None:
        raise ValueError("q_out is given without q")
    for name, t in (("positions", positions), ("q_weight", q_weight), ("k_weight", k_weight)):
        if t is not None:
            named.append((name, t))
    _same_device(device, *named, *given)
    if checked is not None:
        if q_weight is not None or k_weight is not None:
            with _lib._on(stream):
                q_weight, k_weight = _aligned_weight(q_weight), _aligned_weight(k_weight)
        turn = ctypes.byref(_turn_struct(checked, positions, q_weight, k_weight))
    L = _lib.lib()
    st = _lib._call_on(device, stream, L.t2v_paged_append, k.data_ptr(), v.data_ptr(), sk, sv, qp, sq, heads,
                       cu_seqlens.data_ptr(), T, pages._ref, turn, None if q_out is None else q_out.data_ptr())
    if st != _lib.T2V_OK:
        _lib._check(L, st)
    return q_out


def _numbers(x):
    """Page numbers as a contiguous int32 array."""
    x = np.asarray(x)
    if x.dtype != np.int32 and x.size and (x.dtype.kind not in "iu" or x.min() < -2 ** 31 or x.max() >= 2 ** 31):
        raise ValueError(f"src and dst must be page numbers, got {x.dtype} of another kind or range")
    return np.ascontiguousarray(x, dtype=np.int32)


def _buffers(buffers):
    """What t2v_page_copy takes of the buffers, checked: device, addresses, their number, pages, strides and sizes in bytes."""
    first = buffers[0]
    shape, strides, dtype, device = first.shape, first.stride(), first.dtype, first.device
    if len(shape) < 2 or 0 in shape[1:]:
        raise ValueError(f"buffers must be [pages, ...] with pages of a size, got {tuple(shape)}")
    rows = 1
    for size, step in sorted(zip(shape[1:], strides[1:]), key=lambda x: x[1]):
        if size > 1 and step != rows:
            raise ValueError(f"a page's memory must be dense, got strides {strides}")
        rows *= size
    item = first.element_size()
    for b in buffers:
        if b.shape != shape or b.stride() != strides or b.dtype != dtype or b.device != device:
            raise ValueError("buffers must have one shape, strides, dtype and device")
    if not first.is_cuda:
        raise ValueError("buffers must be CUDA tensors")
    ptrs = (ctypes.c_void_p * len(buffers))(*[b.data_ptr() for b in buffers])
    return device, ptrs, len(buffers), shape[0], (strides[0] if shape[0] > 1 else rows) * item, rows * item


def page_copy(buffers, src, dst, stream=None):
    """Copies pages src[i] to pages dst[i] in every one of `buffers`: a tensor [pages, ...] on the GPU or a sequence of them, of one shape and
    strides, each page's memory dense and apart from the other buffers' pages. src, dst: host int32 arrays; no page may be written twice, nor both read
    and written."""
    import torch
    buffers = (buffers,) if isinstance(buffers, torch.Tensor) else tuple(buffers)
    src, dst = _numbers(src), _numbers(dst)
    if src.ndim != 1 or src.shape != dst.shape:
        raise ValueError("src and dst must be 1-D arrays of one length")
    if buffers:
        _copy(_buffers(buffers), src, dst, stream)


def _copy(buffers, src, dst, stream=None):
    device, *rest = buffers
    L = _lib.lib()
    st = _lib._call_on(device, stream, L.t2v_page_copy, *rest, src.__array_interface__["data"][0], dst.__array_interface__["data"][0],
                       src.shape[0])
    if st != _lib.T2V_OK:
        _lib._check(L, st)


class PagedCache:
    """Keys and values of several layers and many sequences in one paged cache on the GPU. Sequences are numbers, the rows of one table that
    all layers share; every call below takes all of them, those without new tokens with none:

        cache = PagedCache(layers, pages, kv_heads, head_dim)
        s = cache.add()
        cache.extend([s], [prompt_tokens])            # room for its tokens, which count from here on
        paged_append(k, v, cache.layer(0), cu_seqlens)
        out, lse = paged_attn_fwd(q, cache.layer(0), cu_seqlens, scale)
        t = cache.fork(s)                             # shares the pages; the one begun is copied when either goes on

    cu_seqlens (cache.offsets({s: prompt_tokens})) has an entry for every sequence and one more. The bookkeeping is on the host (table:
    PageTable); its changes and the pages' copies are enqueued on the current stream, which the calls on the cache must follow. A captured step reads
    lengths and table on the GPU: reserve() room for its tokens, let the graph add them to ``lengths``, and tell grown() afterwards, before any
    other change. A fork or truncation of a sequence ends its room: reserve() again before the next replay."""

    def __init__(self, layers: int, pages: int, kv_heads: int, head_dim: int, page_size: int = 64, sequences: int = 64, width=None,
                 device="cuda"):
        import torch
        from .page_table import PageTable
        self.host = PageTable(pages, page_size, sequences, pages if width is None else width)
        self.data = torch.zeros((layers, 2, pages, page_size, kv_heads, head_dim), dtype=torch.bfloat16, device=device)
        self.table = torch.full(self.host.table.shape, -1, dtype=torch.int32, device=device)
        self.lengths = torch.zeros(sequences, dtype=torch.int32, device=device)
        self._layers = [Pages(x[0], x[1], self.table, self.lengths) for x in self.data]
        self._buffers = _buffers([y for x in self.data for y in x]) if layers else None
        self._sent = self.host.table.copy()  # what the GPU's table holds
        self._width = 0  # columns of it that may hold pages

    def layer(self, i: int) -> Pages:
        """Layer i's pages, for paged_append and paged_attn_fwd."""
        return self._layers[i]

    @property
    def free_pages(self) -> int:
        return self.host.free_pages

    def offsets(self, tokens):
        """cu_seqlens on the GPU for a call in which sequence s has tokens[s] new tokens (a dict, or one count for each sequence)."""
        return self._to_device(self._host().offsets(tokens))

    def _to_device(self, x, out=None):
        import torch
        host = torch.from_numpy(x).pin_memory()  # a new pinned tensor: its memory is not reused before the copy has run
        return host.to(self.data.device, non_blocking=True) if out is None else out.copy_(host, non_blocking=True)

    def _host(self):
        """The bookkeeping, for a change of it."""
        import torch
        if self.data.is_cuda and torch.cuda.is_current_stream_capturing():
            raise RuntimeError("a captured graph cannot hand out or free pages, nor take offsets: reserve() room and make them before the capture")
        return self.host

    def _sync(self, pairs=None, lengths=True):
        if pairs is not None and pairs[0].size and self._buffers is not None:
            _copy(self._buffers, *pairs)
        width = max(self._width, int(self.host.counts.max()))
        now, sent = self.host.table[:, :width], self._sent[:, :width]
        if not np.array_equal(now, sent):
            self._to_device(np.ascontiguousarray(now), self.table[:, :width])
            sent[:] = now
        self._width = int(self.host.counts.max())
        if lengths:
            self._to_device(self.host.lengths, self.lengths)

    def add(self) -> int:
        """A new, empty sequence's number."""
        return self._host().add()

    def extend(self, sequences, tokens) -> None:
        """Room for so many new tokens in each of the sequences (numbers), which count in their lengths from here on. Raises RuntimeError,
        and changes nothing, if there are not enough pages."""
        self._sync(self._host().extend(sequences, tokens))

    def reserve(self, sequences, tokens) -> None:
        """Room for so many new tokens that a captured step will add to the lengths by itself."""
        self._sync(self._host().reserve(sequences, tokens), lengths=False)

    def grown(self, sequences, tokens) -> None:
        """Tells of tokens that were added to the lengths on the GPU."""
        self._host().grown(sequences, tokens)

    def fork(self, sequence: int) -> int:
        """A new sequence with the same tokens; both share the pages."""
        s = self._host().fork(sequence)
        self._sync()
        return s

    def free(self, sequence: int) -> None:
        """Ends a sequence."""
        self._host().free(sequence)
        self._sync()

    def truncate(self, sequence: int, tokens: int) -> None:
        """Takes a sequence back to its first tokens."""
        self._host().truncate(sequence, tokens)
        self._sync()

    def compact(self) -> int:
        """Moves pages so that those in use are the first; returns how many moved."""
        pairs = self._host().compact()
        self._sync(pairs)
        return int(pairs[0].size)
