"""libt2vattn: packed variable-length attention (bidirectional, and causal with grouped heads; forward and
backward), causal attention over a paged cache of keys and values, norms and rotary positions for AMD MI355X (gfx950), behind a C ABI
(include/t2vattn.h).

The binding below only marshals arguments; all computation is in the HIP library.
"""
from ._lib import (  # noqa: F401
    ORDER_LONGEST_FIRST, ORDER_NATURAL, T2VError, attn_bwd, attn_fwd, causal_attn_bwd, causal_attn_fwd, t2v_attn_bwd, t2v_attn_fwd,
    t2v_build_worklist, t2v_kernel_times, t2v_last_error, t2v_timing_enable, t2v_plan_makespan, t2v_release_cache, t2v_version,
    use_checked_library,
)
from .autograd import varlen_attention, varlen_causal_attention  # noqa: F401
from .norm_rotary import norm_rotary, norm_rotary_apply, norm_rotary_bwd  # noqa: F401
from .paged import PagedCache, Pages, page_copy, paged_append, paged_attn_fwd  # noqa: F401
from .rotary import rotary, rotary_apply, rotary_frequencies  # noqa: F401
