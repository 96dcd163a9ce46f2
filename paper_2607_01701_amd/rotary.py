"""Rotary positions for q and k (t2v_rotary): frequencies, the call, and its autograd wrapper. The
binding marshals arguments; the computation is in the HIP library."""
from __future__ import annotations

import ctypes
import math

import numpy as np

from . import _lib
from .autograd import check_capture, note_leaves

LAYOUTS = {"half": 0, "interleaved": 1}
SCALINGS = (None, "linear", "ntk", "yarn")
_SECTIONS = {n: ctypes.c_int32 * n for n in (1, 2, 3)}


def rotary_frequencies(sections, theta: float = 10000.0, scaling=None, factor: float = 1.0, trained=None,
                       slow: float = 1.0, fast: float = 32.0):
    """Frequencies (float64, radians a position) and the factor on the turned dimensions, for rotary().

    sections: pairs of dimensions turned (an int), or pairs for each axis of the positions (up to three, e.g.
    frame, row and column of a latent patch). Pair j of n turns by theta^(-j / n) a position. To reach
    ``factor`` times the ``trained`` positions:
      "linear"  positions shrink by the factor;
      "ntk"     theta grows by factor^(n / (n - 1)), so that the slowest pair shrinks by the factor and the
                fastest not at all;
      "yarn"    pairs that turn at least ``fast`` times over the trained positions stay, those that turn at
                most ``slow`` times shrink by the factor, with a ramp between, and the turned dimensions
                are multiplied by 0.1 ln(factor) + 1 (Peng et al. 2023, arXiv:2309.00071)."""
    sections = (sections,) if isinstance(sections, int) else tuple(sections)
    if not 1 <= len(sections) <= 3 or any(n < 0 for n in sections) or sum(sections) < 1:
        raise ValueError(f"sections must be one to three counts of pairs, got {sections}")
    if scaling not in SCALINGS:
        raise ValueError(f"scaling must be one of {SCALINGS}, got {scaling!r}")
    if not (math.isfinite(theta) and theta > 0 and math.isfinite(factor) and factor > 0):
        raise ValueError("theta and factor must be positive")
    if scaling == "yarn" and (trained is None or not trained > 0 or not 0 < slow < fast):
        raise ValueError("yarn needs the trained positions and 0 < slow < fast")
    freqs = []
    for n in sections:
        base = theta * factor ** (n / (n - 1)) if scaling == "ntk" and n > 1 else theta
        f = base ** -(np.arange(n, dtype=np.float64) / max(n, 1))
        if scaling == "linear":
            f = f / factor
        elif scaling == "yarn":
            keep = np.clip((trained * f / (2 * np.pi) - slow) / (fast - slow), 0.0, 1.0)
            f = f * keep + f / factor * (1.0 - keep)
        freqs.append(f)
    return np.concatenate(freqs), 0.1 * math.log(factor) + 1.0 if scaling == "yarn" and factor > 1.0 else 1.0


def rotary_apply(q, k, positions, freqs, layout: str = "half", sections=None, mscale: float = 1.0,
                 inverse: bool = False, q_out=None, k_out=None, stream=None):
    """q [T, H, D] and k [T, Hk, D] (either may be None) turned by their positions: bf16 on the GPU, tokens any
    distance apart (slices of a fused projection), D 64 or 128. positions: int32 on the GPU, [T], or [axes, T]
    with ``sections`` counting the pairs of each axis. The first 2 len(freqs) dimensions turn, in pairs
    (j, j + len(freqs)) ("half") or (2 j, 2 j + 1) ("interleaved"), and are multiplied by mscale; the others are
    copied. inverse turns back by the same angles (the gradient). Returns contiguous (q, k)."""
    args = _arguments(q, k, positions, freqs, layout, sections, mscale)
    return _turn(q, k, positions, args, inverse, q_out, k_out, stream)


def _arguments(q, k, positions, freqs, layout, sections, mscale):
    """Checks all but the layout of q's and k's tokens; returns what the library takes besides tensors."""
    first = q if q is not None else k
    if first is None:
        raise ValueError("q and k are both None")
    if any(x is not None and x.dim() != 3 for x in (q, k)):
        raise ValueError("q and k must be [tokens, heads, head_dim]")
    if layout not in LAYOUTS:
        raise ValueError(f"layout must be one of {tuple(LAYOUTS)}, got {layout!r}")
    T = first.shape[0]
    f = freqs
    if type(f) is not np.ndarray or f.dtype != np.float64 or not f.flags.c_contiguous:
        f = np.ascontiguousarray(freqs, dtype=np.float64)
    if f.ndim != 1:
        raise ValueError("freqs must be a 1-D array, one frequency a pair")
    pairs = f.shape[0]
    sections = (pairs,) if sections is None else tuple(sections)
    n_sec = len(sections)
    if not 1 <= n_sec <= 3 or sum(sections) != pairs:
        raise ValueError(f"sections {sections} are not one to three counts that sum to the {pairs} frequencies")
    _check_positions(positions, n_sec, T)
    return f, _SECTIONS[n_sec](*sections), n_sec, LAYOUTS[layout], float(mscale)


def _check_positions(positions, axes, T):
    import torch
    if positions.shape != (axes, T) and (axes > 1 or positions.shape != (T,)):
        raise ValueError(f"positions has shape {tuple(positions.shape)}, expected {(axes, T)}")
    if positions.dtype != torch.int32 or not positions.is_contiguous():
        raise ValueError("positions must be contiguous int32")


def _turn(q, k, positions, args, inverse, q_out=None, k_out=None, stream=None):
    import torch
    first = q if q is not None else k
    T, _, D = first.shape
    named, specs, ins = [("positions", positions)], [], []
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
    _lib._check_on_device(named)
    outs, given = _lib._outputs(specs, first.device, stream)
    if given:
        _lib._check_on_device((named[0], *given))
    q_out = outs[0] if q is not None else None
    k_out = outs[-1] if k is not None else None
    (qp, sq, heads), (kp, sk, kv_heads) = ins
    f, sections, n_sec, layout, mscale = args
    L = _lib.lib()
    st = _lib._call_on(first.device, stream, L.t2v_rotary, qp, kp, sq, sk, positions.data_ptr(), T, heads, kv_heads, D,
                       f.__array_interface__["data"][0], sections, n_sec, layout, mscale, 1 if inverse else 0,
                       None if q_out is None else q_out.data_ptr(), None if k_out is None else k_out.data_ptr())
    if st != _lib.T2V_OK:
        _lib._check(L, st)
    return q_out, k_out


def _function():
    import torch

    class _Rotary(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, positions, args, inverse):
            out = _turn(q, k, positions, args, inverse)
            note_leaves(ctx, q, k)
            ctx.save_for_backward(positions)
            ctx.args, ctx.inverse = args, inverse
            ctx.set_materialize_grads(False)
            return out

        @staticmethod
        def backward(ctx, dq, dk):
            if dq is None and dk is None:
                return (None,) * 5
            check_capture(ctx)
            (positions,) = ctx.saved_tensors
            _check_positions(positions, ctx.args[2], (dk if dq is None else dq).shape[0])  # a hook may have changed them
            # R(angle) transposed is R(-angle); with create_graph, the turn back has a gradient of its own.
            dq, dk = (x if x is None or _rows(x) else _lib._aligned(x) for x in (dq, dk))
            turn = _Rotary.apply if torch.is_grad_enabled() else _turn
            return (*turn(dq, dk, positions, ctx.args, not ctx.inverse), None, None, None)

    return _Rotary


def _rows(t) -> bool:
    """Whether the call takes t as it is: each token's heads contiguous, tokens at least a token apart."""
    T, H, D = t.shape
    return t.data_ptr() % 16 == 0 and (t.is_contiguous() or (
        t.stride(2) == 1 and t.stride(1) == D and H * D <= t.stride(0) <= 1 << 22 and t.stride(0) % 8 == 0))


_FN = None


def rotary(q, k, positions, freqs, layout: str = "half", sections=None, mscale: float = 1.0):
    """rotary_apply with autograd: gradients flow to q and k (either may be None), and have gradients of their own.
    Forward-mode derivatives are refused."""
    import torch
    from torch.autograd.forward_ad import unpack_dual
    grads = torch.is_grad_enabled()
    if not any(x is not None and (grads and x.requires_grad or unpack_dual(x).tangent is not None) for x in (q, k)):
        return rotary_apply(q, k, positions, freqs, layout, sections, mscale)
    global _FN
    if _FN is None:
        _FN = _function()
    args = _arguments(q, k, positions, np.array(freqs, dtype=np.float64, copy=True), layout, sections, mscale)
    return _FN.apply(q, k, positions, args, False)
