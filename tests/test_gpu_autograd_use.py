"""The autograd wrappers as programs use them: saved tensors that hooks move or copy, and gradients as other operations
leave them."""
import numpy as np
import pytest
import torch

import paper_2607_01701_amd as t2v

from gpu_util import log

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def cu(lengths):
    return np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)


def rand(*shape, seed=0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).bfloat16().cuda()


def saved_on_cpu():
    return torch.autograd.graph.save_on_cpu()


def saved_dense():
    return torch.autograd.graph.saved_tensors_hooks(lambda x: x.clone(memory_format=torch.contiguous_format), lambda x: x)


@pytest.mark.parametrize("hooks", [saved_on_cpu, saved_dense])
@pytest.mark.parametrize("H,Hk,D", [(6, 2, 128), (3, 1, 64)])
def test_gradients_under_saved_tensor_hooks(H, Hk, D, hooks):
    """Slices of a fused projection, saved as dense copies: the gradients are those without hooks, bitwise."""
    log(f"case hooks {hooks.__name__} {H}/{Hk}x{D}")
    n = [300, 77]
    w = rand(377, H + 2 * Hk, D, seed=1).requires_grad_(True)
    g, pos = rand(377, H, D, seed=2), torch.arange(377, dtype=torch.int32, device="cuda")
    freqs, _ = t2v.rotary_frequencies(D // 2)

    def gradients():
        q, k = t2v.rotary(w[:, :H], w[:, H:H + Hk], pos, freqs)
        out, _ = t2v.varlen_causal_attention(q, k, w[:, H + Hk:], cu(n), 0.1)
        plain, _ = t2v.varlen_causal_attention(w[:, :H], w[:, H:H + Hk], w[:, H + Hk:], cu(n), 0.1)
        return out + plain

    (want,) = torch.autograd.grad(gradients(), w, g)
    with hooks():
        out = gradients()
    (got,) = torch.autograd.grad(out, w, g)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.isfinite(want.float()).all() and (want != 0).any()


@pytest.mark.parametrize("H,Hk,D", [(4, 2, 128), (2, 2, 64)])
def test_gradients_of_parts_of_a_concatenation(H, Hk, D):
    """They start at any even address: the results are those of aligned ones, bitwise."""
    log(f"case unaligned gradients {H}/{Hk}x{D}")
    n = [70, 9]
    q, k, v = (rand(79, h, D, seed=h).requires_grad_(True) for h in (H, Hk, Hk))
    pos = torch.arange(79, dtype=torch.int32, device="cuda")
    freqs, _ = t2v.rotary_frequencies(D // 2)

    def outputs():
        a, b = t2v.rotary(q, k, pos, freqs, "interleaved")
        o, _ = t2v.varlen_causal_attention(q, k, v, cu(n), 0.1)
        outs = [a, b, o]
        if H == Hk:
            outs.append(t2v.varlen_attention(q, k, v, cu(n), 0.1)[0])
        return outs

    outs = outputs()
    sizes = [o.numel() for o in outs]
    whole = rand(sum(sizes) + len(sizes), seed=9)
    want = torch.autograd.grad(outs, (q, k, v), [p.clone().view(o.shape) for p, o in zip(
        (x[1:] for x in whole.split([s + 1 for s in sizes])), outs)])
    one = torch.zeros(1, dtype=torch.bfloat16, device="cuda")
    joined = torch.cat([x for o in outputs() for x in (one, o.flatten())])
    got = torch.autograd.grad(joined, (q, k, v), whole)
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("name", ["bidirectional", "causal", "rotary"])
def test_capture_after_a_warm_up_whose_outputs_are_kept(name):
    """The eager graph of a side stream, still alive, does not hinder the capture of a training step on another stream; replays
    give the eager gradients, with eager steps between them."""
    log(f"case capture beside a warm-up, {name}")
    n = [200, 30]
    q, k, v = (rand(230, 2, 64, seed=i).requires_grad_(True) for i in (1, 2, 3))
    g = rand(230, 2, 64, seed=9)
    pos = torch.arange(230, dtype=torch.int32, device="cuda")
    freqs, _ = t2v.rotary_frequencies(32)

    def step():
        if name == "rotary":
            a, b = t2v.rotary(q, k, pos, freqs)
            return a + b
        return (t2v.varlen_attention if name == "bidirectional" else t2v.varlen_causal_attention)(q, k, v, cu(n), 0.1)[0]

    leaves = (q, k) if name == "rotary" else (q, k, v)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        kept = step()
        want = torch.autograd.grad(kept, leaves, g, retain_graph=True)
    torch.cuda.synchronize()
    want = [x.clone() for x in want]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = torch.autograd.grad(step(), leaves, g)
    for i in range(3):
        for x in got:
            x.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i
        with torch.cuda.stream(side):
            eager = torch.autograd.grad(step(), leaves, g)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, want)), i
    assert kept.requires_grad
