"""More refusals of the rotary call on the CPU: outputs without their tensor, more tokens than a launch takes."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2607_01701_amd as t2v
from paper_2607_01701_amd import _lib


@pytest.mark.parametrize("given,out", [("q", "k_out"), ("k", "q_out")])
def test_an_output_without_its_tensor(given, out):
    x = torch.zeros(9, 2, 64, dtype=torch.bfloat16)
    a = {"q": None, "k": None, given: x}
    with pytest.raises(ValueError, match=f"{out} is given without"):
        t2v.rotary_apply(a["q"], a["k"], torch.zeros(9, dtype=torch.int32), np.ones(8), **{out: torch.zeros_like(x)})


@pytest.mark.parametrize("tokens,heads,head_dim,pairs", [(1 << 29, 1, 128, 64), ((1 << 31) - 1, 2, 64, 32), (1 << 28, 120, 64, 3)])
def test_more_workgroups_than_a_launch_takes(tokens, heads, head_dim, pairs):
    """A launch counts its threads in 32 bits. (Addresses are never read.)"""
    a, f, n = 1 << 20, np.ones(pairs), np.array([pairs], dtype=np.int32)
    L = _lib.lib()
    st = L.t2v_rotary(None, a, 0, heads * head_dim, a + (1 << 60), tokens, 0, heads, head_dim, f.ctypes.data,
                      n.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)), 1, 0, 1.0, 0, None, a + (1 << 50), None)
    assert st == _lib.T2V_ERR_INVALID_ARG and "workgroups" in _lib.t2v_last_error(L), _lib.t2v_last_error(L)
