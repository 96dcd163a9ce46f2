"""What the autograd wrappers pass to the library, on the CPU with the library's calls replaced by ones that note
their arguments and launch nothing."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2607_01701_amd as t2v
from paper_2607_01701_amd import _lib

CU = np.array([0, 30, 50], dtype=np.int32)


class Calls:
    """Stands for the library: each call is noted with its arguments and succeeds."""

    def __init__(self):
        self.made = []

    def __getattr__(self, name):
        def call(*args):
            self.made.append((name, args))
            return _lib.T2V_OK
        return call

    def args(self, name):
        (found,) = [a for n, a in self.made if n == name]
        return found


@pytest.fixture
def calls(monkeypatch):
    c = Calls()
    monkeypatch.setattr(_lib, "lib", lambda: c)
    monkeypatch.setattr(_lib, "_check_on_device", lambda named: None)
    monkeypatch.setattr(_lib, "_call_on", lambda device, stream, fn, *args: fn(*args, None))
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 0, raising=False)
    return c


def dense(x):
    return x.clone(memory_format=torch.contiguous_format)


def address(x):
    return getattr(x, "value", x)


HOOKS = [None, (dense, lambda x: x), (lambda x: x, dense)]


@pytest.mark.parametrize("hooks", HOOKS, ids=["none", "pack", "unpack"])
def test_causal_backward_describes_the_tensors_that_it_passes(calls, hooks):
    """Saved-tensor hooks (offloading, compression) may give dense copies of slices of a fused projection."""
    H, Hk, D = 6, 2, 128
    w = torch.zeros(50, H + 2 * Hk, D, dtype=torch.bfloat16).requires_grad_(True)
    q, k, v = w[:, :H], w[:, H:H + Hk], w[:, H + Hk:]
    seen = {}

    def unpacked(x):
        y = hooks[1](x)
        seen[y.data_ptr()] = y
        return y

    if hooks is None:
        out, _ = t2v.varlen_causal_attention(q, k, v, CU, 0.1)
        seen.update({x.data_ptr(): x for x in (q, k, v)})
    else:
        with torch.autograd.graph.saved_tensors_hooks(hooks[0], unpacked):
            out, _ = t2v.varlen_causal_attention(q, k, v, CU, 0.1)
    out.backward(torch.zeros_like(out))
    a = calls.args("t2v_causal_bwd")
    for pointer, stride, heads in zip(a[:3], a[3:6], (H, Hk, Hk)):
        x = seen[address(pointer)]
        assert x.shape == (50, heads, D) and x.stride() == (stride, D, 1)
    assert [ctypes.c_int(n).value for n in a[10:14]] == [2, H, Hk, D]


@pytest.mark.parametrize("name,change", [
    ("q", lambda x: x[:-1]), ("k", lambda x: x.float()), ("v", lambda x: x.transpose(0, 1).contiguous().transpose(0, 1)),
    ("out", lambda x: x.transpose(0, 1).contiguous().transpose(0, 1)), ("lse", lambda x: x.double()),
    ("lse", lambda x: x.t().contiguous().t()),
])
def test_causal_backward_refuses_what_a_hook_changed(calls, name, change):
    H, Hk, D = 4, 2, 64
    q, k, v = (torch.zeros(50, h, D, dtype=torch.bfloat16).requires_grad_(True) for h in (H, Hk, Hk))
    order = iter(("q", "k", "v", "out", "lse"))
    with torch.autograd.graph.saved_tensors_hooks(lambda x: (next(order), x), lambda p: change(p[1]) if p[0] == name else p[1]):
        out, _ = t2v.varlen_causal_attention(q, k, v, CU, 0.1)
    with pytest.raises(ValueError, match=f"{name} "):
        out.backward(torch.zeros_like(out))
    assert "t2v_causal_bwd" not in [n for n, _ in calls.made]


@pytest.mark.parametrize("change,msg", [
    (lambda x: x.long(), "int32"), (lambda x: x[:, :-1], "shape"), (lambda x: x.t().contiguous().t(), "contiguous"),
])
def test_rotary_backward_refuses_positions_that_a_hook_changed(calls, change, msg):
    q = torch.zeros(50, 4, 64, dtype=torch.bfloat16).requires_grad_(True)
    positions = torch.zeros(2, 50, dtype=torch.int32)
    with torch.autograd.graph.saved_tensors_hooks(lambda x: x, change):
        out, _ = t2v.rotary(q, None, positions, np.ones(32), sections=(16, 16))
    with pytest.raises(ValueError, match=f"positions.*{msg}"):
        out.backward(torch.zeros_like(out))
    assert len(calls.made) == 1


@pytest.mark.parametrize("grad", [True, False], ids=["grad", "no_grad"])
@pytest.mark.parametrize("which", ["q", "k", "attention"])
def test_forward_mode_derivatives_are_refused(calls, which, grad):
    """A tangent that the calls do not carry on is not dropped in silence; without one, a dual level changes nothing."""
    x = torch.zeros(50, 4, 64, dtype=torch.bfloat16)
    positions = torch.zeros(50, dtype=torch.int32)
    with torch.autograd.forward_ad.dual_level(), torch.set_grad_enabled(grad):
        assert t2v.rotary(x, x, positions, np.ones(32))[0].shape == x.shape
        dual = torch.autograd.forward_ad.make_dual(x, torch.ones_like(x))
        with pytest.raises((RuntimeError, NotImplementedError), match="jvp"):
            if which == "attention":
                t2v.varlen_causal_attention(dual, x, x, CU, 0.1)
            else:
                t2v.rotary(dual if which == "q" else None, dual if which == "k" else x, positions, np.ones(32))


@pytest.mark.parametrize("which", ["bidirectional", "causal", "rotary", "rotary k"])
def test_gradients_at_any_address(calls, which):
    """The gradient of a concatenation's part is contiguous and may start anywhere; the library takes 16-byte addresses."""
    x = torch.zeros(50, 4, 64, dtype=torch.bfloat16).requires_grad_(True)
    if which.startswith("rotary"):
        both = (x, None) if which == "rotary" else (None, x)
        out = [y for y in t2v.rotary(*both, torch.zeros(50, dtype=torch.int32), np.ones(32)) if y is not None][0]
    else:
        out, _ = (t2v.varlen_attention if which == "bidirectional" else t2v.varlen_causal_attention)(x, x, x, CU, 0.1)
    g = torch.zeros(out.numel() + 1, dtype=out.dtype)[1:].view(out.shape)
    assert g.is_contiguous() and g.data_ptr() % 16 == 2
    out.backward(g)
    name, place = {"bidirectional": ("t2v_attn_bwd", 10), "causal": ("t2v_causal_bwd", 15), "rotary": ("t2v_rotary", 0),
                   "rotary k": ("t2v_rotary", 1)}[which]
    a = [args for n, args in calls.made if n == name][-1]
    assert a[place] != 0 and a[place] % 16 == 0


def attend(name, q, k, v):
    if name == "rotary":
        return t2v.rotary(q, k, torch.zeros(50, dtype=torch.int32), np.ones(32))[0]
    return (t2v.varlen_attention if name == "bidirectional" else t2v.varlen_causal_attention)(q, k, v, CU, 0.1)[0]


@pytest.mark.parametrize("name", ["bidirectional", "causal", "rotary"])
@pytest.mark.parametrize("eager,refused", [(0, True), (7, False), (9, False), (None, False)],
                         ids=["default stream", "side stream", "the capture's stream", "no eager graph"])
def test_captured_backward_beside_an_eager_graph(calls, monkeypatch, name, eager, refused):
    """Only a leaf whose gradient node was made on the default stream cannot be captured: any other stream may
    join a capture, as that of a warm-up whose outputs are still there."""
    q, k, v = (torch.zeros(50, 4, 64, dtype=torch.bfloat16).requires_grad_(True) for _ in range(3))
    current = [eager or 0]
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: current[0], raising=False)
    alive = attend(name, q, k, v) if eager is not None else None
    current[0] = 9
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    out = attend(name, q, k, v)
    g = torch.zeros_like(out)
    if refused:
        with pytest.raises(RuntimeError, match="default stream"):
            out.backward(g)
    else:
        out.backward(g)
    if refused:  # until the eager graph is gone
        del alive, out
        attend(name, q, k, v).backward(g)


@pytest.mark.parametrize("name", ["bidirectional", "causal", "rotary"])
def test_calls_without_a_gpu_name_the_tensor(name, monkeypatch):
    """The refusal of tensors that are not on a GPU comes before any question about streams."""
    def none(*_):
        raise RuntimeError("no GPU")
    for place in ("current_device", "current_stream"):
        monkeypatch.setattr(torch.cuda, place, none)
    q, k, v = (torch.zeros(50, 4, 64, dtype=torch.bfloat16).requires_grad_(True) for _ in range(3))
    with pytest.raises(ValueError, match="must be a CUDA tensor"):
        attend(name, q, k, v)
