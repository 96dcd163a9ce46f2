"""Norms of the heads of q and k with rotary positions after them (t2v_norm_rotary), and their autograd wrapper. The
binding marshals arguments; the computation is in the HIP library."""
from __future__ import annotations

import ctypes
import math

import numpy as np

from . import _lib
from .autograd import check_capture, note_leaves
from .rotary import _arguments, _check_positions, _rows


def _weights(q_weight, k_weight, q, k, eps):
    """Checks the norm's weights and eps; returns whether the weights are float32."""
    import torch
    if eps is not None and not (math.isfinite(eps) and eps >= 0.0):
        raise ValueError(f"eps must be finite and >= 0 (None: no norm), got {eps}")
    f32 = None
    for w, x, name in ((q_weight, q, "q"), (k_weight, k, "k")):
        if w is None:
            continue
        if eps is None or x is None:
            raise ValueError(f"{name}_weight is given without " + ("a norm (eps)" if eps is None else name))
        if w.shape != (x.shape[2],) or w.dtype not in (torch.float32, torch.bfloat16):
            raise ValueError(f"{name}_weight must be [{x.shape[2]}] in float32 or bfloat16, got {tuple(w.shape)} in {w.dtype}")
        if f32 is not None and f32 != (w.dtype == torch.float32):
            raise ValueError("q_weight and k_weight must have the same dtype")
        f32 = w.dtype == torch.float32
    return bool(f32)


def _checked(q, k, positions, freqs, layout, sections, mscale, q_weight, k_weight, eps):
    """All but the layout of the tokens; returns what _turn_struct takes besides tensors."""
    if freqs is None:
        first = q if q is not None else k
        if first is None:
            raise ValueError("q and k are both None")
        if any(x is not None and x.dim() != 3 for x in (q, k)):
            raise ValueError("q and k must be [tokens, heads, head_dim]")
        if positions is not None or sections is not None:
            raise ValueError("positions or sections are given without freqs")
        args = None
    elif positions is None:
        raise ValueError("freqs are given without positions")
    else:
        args = _arguments(q, k, positions, freqs, layout, sections, mscale)
    return args, _weights(q_weight, k_weight, q, k, eps), eps


def _turn_struct(checked, positions, q_weight, k_weight):
    args, f32, eps = checked
    t = _lib.Turn()
    if args is not None:
        t.positions = positions.data_ptr()
        t.freqs = args[0].__array_interface__["data"][0]
        t.sections = ctypes.addressof(args[1])
        t.n_sections, t.layout, t.mscale = args[2], args[3], args[4]
    t.eps = -1.0 if eps is None else eps
    if q_weight is not None:
        t.q_weight = q_weight.data_ptr()
    if k_weight is not None:
        t.k_weight = k_weight.data_ptr()
    t.weights_f32 = f32
    return t


def norm_rotary_apply(q, k, positions, freqs, q_weight=None, k_weight=None, eps=1e-6, layout: str = "half", sections=None,
                      mscale: float = 1.0, q_out=None, k_out=None, stream=None):
    """The heads of q [T, H, D] and k [T, Hk, D] divided by their root mean square (eps added to the mean square), times q_weight and
    k_weight ([D], both float32 or both bfloat16; None: ones), then turned as by rotary_apply, in one pass rounded once. bf16 on
    the GPU, tokens any distance apart, either may be None; eps None: no norm; freqs (and positions) None: no turn. Returns contiguous (q, k),
    without gradients or tangents, whatever the arguments have: norm_rotary is the call with autograd."""
    checked = _checked(q, k, positions, freqs, layout, sections, mscale, q_weight, k_weight, eps)
    return _forward(q, k, positions, checked, q_weight, k_weight, q_out, k_out, stream)


def _aligned_weight(w):
    return w if w is None else _lib._aligned(w)


def _forward(q, k, positions, checked, q_weight, k_weight, q_out=None, k_out=None, stream=None):
    import torch
    first = q if q is not None else k
    T, _, D = first.shape
    named = [] if positions is None else [("positions", positions)]
    specs, ins = [], []
    for x, o, name in ((q, q_out, "q"), (k, k_out, "k")):
        if x is None:
            if o is not None:
                raise ValueError(f"{name}_out is given without {name}")
            ins.append((None, 0, 0))
            continue
        shape = (T, x.shape[1], D)
        step = _lib._check_rows(x, name, shape)
        named.append((name, x))
        specs.append((name + "_out", o, shape, torch.bfloat16))
        ins.append((x.data_ptr(), step, shape[1]))
    named += [(n, w) for n, w in (("q_weight", q_weight), ("k_weight", k_weight)) if w is not None]
    _lib._check_on_device(named)
    outs, given = _lib._outputs(specs, first.device, stream)
    if given:
        _lib._check_on_device((named[0], *given))
    q_out = outs[0] if q is not None else None
    k_out = outs[-1] if k is not None else None
    (qp, sq, heads), (kp, sk, kv_heads) = ins
    with _lib._on(stream):
        q_weight, k_weight = _aligned_weight(q_weight), _aligned_weight(k_weight)
    turn = _turn_struct(checked, positions, q_weight, k_weight)
    L = _lib.lib()
    st = _lib._call_on(first.device, stream, L.t2v_norm_rotary, qp, kp, sq, sk, T, heads, kv_heads, D, ctypes.byref(turn),
                       None if q_out is None else q_out.data_ptr(), None if k_out is None else k_out.data_ptr())
    if st != _lib.T2V_OK:
        _lib._check(L, st)
    return q_out, k_out


def norm_rotary_bwd(q, k, dq_out, dk_out, positions, freqs, q_weight=None, k_weight=None, eps: float = 1e-6,
                    layout: str = "half", sections=None, mscale: float = 1.0, stream=None):
    """Backward of norm_rotary_apply: from its inputs and the gradients of its outputs (tokens any distance apart), those of q and k (bf16) and of
    the weights (of their type, None without weights): (dq, dk, dq_weight, dk_weight), which have no gradients themselves."""
    if eps is None:
        raise ValueError("the backward pass needs a norm; a turn alone is rotary_apply's inverse")
    checked = _checked(q, k, positions, freqs, layout, sections, mscale, q_weight, k_weight, eps)
    return _backward(q, k, dq_out, dk_out, positions, checked, q_weight, k_weight, (True, True), stream)


def _backward(q, k, dq_out, dk_out, positions, checked, q_weight, k_weight, wanted, stream=None):
    """wanted: whether the gradients of q's and k's weights are."""
    import torch
    first = q if q is not None else k
    T, _, D = first.shape
    named = [] if positions is None else [("positions", positions)]
    ins, specs = [], []
    for x, g, w, name in ((q, dq_out, q_weight, "q"), (k, dk_out, k_weight, "k")):
        if (x is None) != (g is None):
            raise ValueError(f"{name} and d{name}_out must both be given")
        if x is None:
            ins.append((None, None, 0, 0, 0))
            continue
        shape = (T, x.shape[1], D)
        ins.append((x.data_ptr(), g.data_ptr(), _lib._check_rows(x, name, shape), _lib._check_rows(g, f"d{name}_out", shape), shape[1]))
        named += [(name, x), (f"d{name}_out", g)]
        specs.append((f"d{name}", None, shape, torch.bfloat16))
    weights = [w if w is not None and x is not None else None for w, x in ((q_weight, q), (k_weight, k))]
    named += [(n, w) for n, w in zip(("q_weight", "k_weight"), weights) if w is not None]
    _lib._check_on_device(named)
    for i, w in enumerate(weights):
        if w is not None and wanted[i]:
            specs.append((("dq_weight", "dk_weight")[i], None, (D,), w.dtype))
    outs, _ = _lib._outputs(specs, first.device, stream)
    by = dict(zip((s[0] for s in specs), outs))
    out = [by.get(n) for n in ("dq", "dk", "dq_weight", "dk_weight")]
    with _lib._on(stream):
        weights = [_aligned_weight(w) for w in weights]
    turn = _turn_struct(checked, positions, *weights)
    (qp, gqp, sq, gsq, heads), (kp, gkp, sk, gsk, kv_heads) = ins
    L = _lib.lib()
    ptrs = [None if o is None else o.data_ptr() for o in out]
    if out[2] is None and out[3] is None:
        st = _lib._call_on(first.device, stream, L.t2v_norm_rotary_bwd, qp, kp, sq, sk, gqp, gkp, gsq, gsk, T, heads, kv_heads,
                           D, ctypes.byref(turn), *ptrs, None, 0, None)
        if st != _lib.T2V_OK:
            _lib._check(L, st)
    else:
        _lib._call_with_workspace(L, L.t2v_norm_rotary_bwd, first.device, stream, qp, kp, sq, sk, gqp, gkp, gsq, gsk, T, heads,
                                  kv_heads, D, ctypes.byref(turn), *ptrs)
    return tuple(out)


def _function():
    import torch
    from torch.autograd.function import once_differentiable

    def gradients(ctx, dq, dk):
        none = (None,) * 6
        if dq is None and dk is None:
            return none
        check_capture(ctx)
        q, k, q_weight, k_weight, positions = ctx.saved_tensors
        # Saved-tensor hooks may give other tensors than the forward pass checked.
        args, f32, eps = ctx.checked
        first = q if q is not None else k
        if args is not None:
            _check_positions(positions, args[2], first.shape[0])
        if _weights(q_weight, k_weight, q, k, eps) != f32:
            raise ValueError("the saved weights have another dtype than in the forward pass")
        dq, dk = (x if x is None or _rows(x) else _lib._aligned(x) for x in (dq, dk))
        q, k = (x if g is not None else None for x, g in ((q, dq), (k, dk)))
        d = _backward(q, k, dq, dk, positions, ctx.checked, q_weight if q is not None else None, k_weight if k is not None else None,
                      ctx.needs_input_grad[2:4])
        return (*d, None, None)

    gradients_once = once_differentiable(gradients)

    class _NormRotary(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, q_weight, k_weight, positions, checked):
            out = _forward(q, k, positions, checked, q_weight, k_weight)
            note_leaves(ctx, q, k, q_weight, k_weight)
            ctx.save_for_backward(q, k, q_weight, k_weight, positions)
            ctx.checked = checked
            ctx.set_materialize_grads(False)
            return out

        @staticmethod
        def backward(ctx, dq, dk):
            return (gradients_once if torch.is_grad_enabled() else gradients)(ctx, dq, dk)

    return _NormRotary


_FN = None


def norm_rotary(q, k, positions, freqs, q_weight=None, k_weight=None, eps: float = 1e-6, layout: str = "half", sections=None,
                mscale: float = 1.0):
    """norm_rotary_apply with autograd: gradients flow to q, k and the weights, and have none of their own: asked for, they
    raise, as forward-mode derivatives do. A norm is needed (rotary turns alone)."""
    import torch
    from torch.autograd.forward_ad import unpack_dual
    if eps is None:
        raise ValueError("norm_rotary needs a norm (eps); rotary turns alone")
    grads = torch.is_grad_enabled()
    if not any(x is not None and (grads and x.requires_grad or unpack_dual(x).tangent is not None)
               for x in (q, k, q_weight, k_weight)):
        return norm_rotary_apply(q, k, positions, freqs, q_weight, k_weight, eps, layout, sections, mscale)
    global _FN
    if _FN is None:
        _FN = _function()
    freqs = None if freqs is None else np.array(freqs, dtype=np.float64, copy=True)
    checked = _checked(q, k, positions, freqs, layout, sections, mscale, q_weight, k_weight, float(eps))
    return _FN.apply(q, k, q_weight, k_weight, positions, checked)
