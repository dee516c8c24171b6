"""The Python binding's own checks of the attention operators, on host tensors: no library call is reached."""
import pytest
import torch

from paper_2607_08779_amd import ssq

BF = torch.bfloat16


def test_decode_refuses_a_workspace_whose_bytes_are_not_its_own():
    """An expanded or strided tensor's element count says nothing about the memory behind its address."""
    q, pools = torch.zeros((2, 1, 8, 64), dtype=BF), [torch.zeros((4, 2, 16, 64), dtype=BF) for _ in "kv"]
    table, lens = torch.zeros((2, 2), dtype=torch.int32), torch.ones(2, dtype=torch.int32)
    for bad in (torch.empty(1, dtype=torch.uint8).expand(1 << 20), torch.empty(1 << 21, dtype=torch.uint8)[::2]):
        with pytest.raises(ValueError, match="workspace"):
            ssq.ssq_attention_decode(q, *pools, table, lens, 32, workspace=bad)
