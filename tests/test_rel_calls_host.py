"""CPU checks of calls of include/cnnk_rel.h: what the binding refuses, sizes of workspaces."""
import pytest
import torch

from paper_2503_23186_amd import cnnk, rel

A = 4096          # an address that is never read


def test_a_plan_tensor_of_fewer_bytes_is_refused():
    need = rel.cnnk_rel_plan_bytes(70, 9)
    d = rel.rel_desc(2, 70, 2, 64, cnnk.BF16, 9)
    for plan in (torch.zeros(need - 1, dtype=torch.uint8), torch.zeros(need // 4 - 1), torch.zeros(rel.cnnk_rel_plan_bytes(69, 9), dtype=torch.uint8)):
        with pytest.raises(ValueError):
            rel.cnnk_rel_attention_fwd(d, A, A, plan, None, None, A, A)
        with pytest.raises(ValueError):
            rel.cnnk_rel_attention_bwd(d, A, A, A, A, plan, None, None, A, A, A, A, 1 << 40)
