"""PyTorch autograd wrapper over the C ABI: the forward calls t2v_attn_fwd (or _qk, or t2v_causal_fwd), the
backward t2v_attn_bwd (or _qk, or t2v_causal_bwd) with the saved out and lse, so a training step (the DiT
forward and backward of Fig. 1) can use the library through loss.backward(). Argument
marshalling only; every step runs in the HIP library."""
from __future__ import annotations

import numpy as np

from . import _lib
from ._lib import _aligned, _cu_array, _stream_handle, attn_bwd, attn_fwd


def _leaves(ctx):
    return [n for n, _ in ctx.next_functions if n is not None and type(n).__name__ == "AccumulateGrad"]


def _on_default_stream(device):
    import torch
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)  # as in _stream_handle
    return (torch.cuda.current_stream(device).cuda_stream if raw is None else raw(device.index)) == 0


def note_leaves(ctx, *inputs):
    """Notes, in a Function's forward, whether the gradient nodes of its leaf inputs were first used on the default stream (torch
    keeps a node as long as any autograd graph holds it, and the stream that was current when it was made with it). A node
    that another operation made before is taken for one of this call's stream."""
    leaves = [x for x in inputs if x is not None and x.requires_grad and x.is_leaf]
    if leaves:
        default = _on_default_stream(leaves[0].device)
        for node in _leaves(ctx):
            node.metadata.setdefault("t2v_default_stream", default)  # lives as long as the node


def check_capture(ctx):
    """Refuses, in a Function's backward, to record into a graph the gradient of a leaf whose node an eager call made on the
    default stream and that call's autograd graph still holds: torch would make that stream part of the capture, which ends the
    process when the capture does. (Any other stream joins a capture, and leaves it.)"""
    import torch
    if not torch.cuda.is_current_stream_capturing():
        return
    if any(node.metadata.get("t2v_default_stream", False) for node in _leaves(ctx)):
        raise RuntimeError("a captured backward pass takes the gradient of a leaf tensor that an eager autograd graph, made "
                           "on the default stream, still holds: drop that graph's outputs before the capture, or make them "
                           "on a side stream")


def _function(attn_fwd, attn_bwd, once=False):
    """The autograd Function of attn_fwd(q, k, v, offsets, scale, key offsets) -> out, lse and what attn_bwd(q, k, v, out, lse,
    dout, kept) needs besides; once: gradients of its gradients raise."""
    import torch
    from torch.autograd.function import once_differentiable

    def gradients(ctx, dout, _dlse):
        if dout is None:  # nothing depends on out
            return None, None, None, None, None, None
        check_capture(ctx)
        return (*attn_bwd(*ctx.saved_tensors, _aligned(dout), ctx.kept), None, None, None)

    gradients_once = once_differentiable(gradients)

    class _VarlenAttention(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, v, cu_seqlens, scale, cu_seqlens_k):
            out, lse, ctx.kept = attn_fwd(q, k, v, cu_seqlens, scale, cu_seqlens_k)
            note_leaves(ctx, q, k, v)
            ctx.save_for_backward(q, k, v, out, lse)
            ctx.mark_non_differentiable(lse)
            # lse never has a gradient: without this, every backward call allocates and fills a
            # zero [H, T] tensor for it, one more launch on an idle queue. With the leaner argument
            # checks: 186 -> 149 to 158 us for a training step of 640 tokens, bound by such host work.
            ctx.set_materialize_grads(False)
            return out, lse

        @staticmethod
        def backward(ctx, dout, dlse):
            return (gradients_once if once and torch.is_grad_enabled() else gradients)(ctx, dout, dlse)

    return _VarlenAttention


def _fwd(q, k, v, cu, scale, cu_k):
    return (*attn_fwd(q, k, v, cu, scale, cu_seqlens_k=cu_k), (cu, scale, cu_k))


def _bwd(q, k, v, out, lse, dout, kept):
    cu, scale, cu_k = kept
    return attn_bwd(q, k, v, out, lse, dout, cu, scale, cu_seqlens_k=cu_k)


def _causal_fwd(q, k, v, cu, scale, cu_k):
    import torch
    args = _lib._causal_arguments(q, k, v, cu, cu_k)
    T, H, D = args[:3]
    _lib._check_on_device((("q", q), ("k", k), ("v", v)))
    out = torch.empty((T, H, D), dtype=torch.bfloat16, device=q.device)
    lse = torch.empty((H, T), dtype=torch.float32, device=q.device)
    _lib._causal_fwd(args, q, k, v, scale, out, lse, None)
    return out, lse, (args, scale)


def _causal_bwd(q, k, v, out, lse, dout, kept):
    # Of what the forward pass checked only the offsets still hold: saved-tensor hooks may give other tensors, such as dense
    # copies of slices, so their strides, shapes, types and devices are taken from themselves.
    import torch
    args, scale = kept
    T, H, D, Tk, Hk, _, cq, ck = args
    strides = tuple(_lib._check_rows(x, n, s) for x, n, s in ((q, "q", (T, H, D)), (k, "k", (Tk, Hk, D)), (v, "v", (Tk, Hk, D))))
    for x, n in ((out, "out"), (dout, "dout")):
        _lib._check_tensor(x, n, (T, H, D))
    _lib._check_tensor(lse, "lse", (H, T), torch.float32)
    _lib._check_on_device((("q", q), ("k", k), ("v", v), ("out", out), ("lse", lse), ("dout", dout)))
    args = (T, H, D, Tk, Hk, strides, cq, ck)
    empty, device = torch.empty, q.device
    dq, dk, dv = (empty((t, h, D), dtype=torch.bfloat16, device=device) for t, h in ((T, H), (Tk, Hk), (Tk, Hk)))
    delta_ws = empty((2, H, T), dtype=torch.float32, device=device)
    _lib._causal_bwd(args, q, k, v, out, lse, dout, scale, dq, dk, dv, delta_ws, None)
    return dq, dk, dv


_FN = None  # varlen_attention's Function, made at its first call (torch is imported late)
_CAUSAL_FN = None


def varlen_attention(q, k, v, cu_seqlens, scale: float, cu_seqlens_k=None):
    """Packed variable-length attention with autograd: q [Tq, H, D], k, v [Tk, H, D] bf16 on the
    GPU; cu_seqlens (and cu_seqlens_k for cross-attention) host int32 offsets. Returns (out, lse);
    gradients flow to q, k and v (lse is not differentiated)."""
    global _FN
    if _FN is None:
        _FN = _function(_fwd, _bwd)
    cu = _cu_array(cu_seqlens)
    ck = None if cu_seqlens_k is None else _cu_array(cu_seqlens_k)
    return _FN.apply(q, k, v, np.array(cu, copy=True), float(scale), None if ck is None else np.array(ck, copy=True))


def varlen_causal_attention(q, k, v, cu_seqlens, scale: float, cu_seqlens_k=None):
    """Causal attention with grouped heads and autograd: q [Tq, H, D], k, v [Tk, Hk, D] as in causal_attn_fwd.
    Returns (out, lse); gradients flow to q, k and v (lse is not differentiated), and have none of their own: asked for,
    they raise."""
    global _CAUSAL_FN
    if _CAUSAL_FN is None:
        _CAUSAL_FN = _function(_causal_fwd, _causal_bwd, once=True)
    cu = np.array(_cu_array(cu_seqlens), copy=True)
    ck = None if cu_seqlens_k is None else np.array(_cu_array(cu_seqlens_k), copy=True)
    return _CAUSAL_FN.apply(q, k, v, cu, float(scale), ck)
