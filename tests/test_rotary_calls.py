"""More refusals of the rotary call on the CPU: outputs without their tensor."""
import numpy as np
import pytest
import torch

import paper_2607_01701_amd as t2v


@pytest.mark.parametrize("given,out", [("q", "k_out"), ("k", "q_out")])
def test_an_output_without_its_tensor(given, out):
    x = torch.zeros(9, 2, 64, dtype=torch.bfloat16)
    a = {"q": None, "k": None, given: x}
    with pytest.raises(ValueError, match=f"{out} is given without"):
        t2v.rotary_apply(a["q"], a["k"], torch.zeros(9, dtype=torch.int32), np.ones(8), **{out: torch.zeros_like(x)})
