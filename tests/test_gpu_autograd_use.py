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
