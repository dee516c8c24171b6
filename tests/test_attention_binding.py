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


def reaches_the_library(call):
    """Past the shape checks a host tensor is refused for where it lies."""
    with pytest.raises(ValueError, match="GPU tensors only"):
        call()


def test_one_head_is_contiguous_whatever_its_stride():
    """The stride between heads says nothing where there is one: [heads, tokens, dim] transposed."""
    q, k = torch.zeros((1, 9, 64), dtype=BF).transpose(0, 1), torch.zeros((1, 12, 64), dtype=BF)[:, 2:11].transpose(0, 1)
    starts, pos, rope = torch.zeros(2, dtype=torch.int32), torch.zeros(9, dtype=torch.int32), torch.zeros((4, 64))
    reaches_the_library(lambda: ssq.ssq_attention_prompt(q, k, k, starts))
    reaches_the_library(lambda: ssq.ssq_qk_norm_rope(q, k, pos, rope))
    pools, table = [torch.zeros((4, 1, 16, 64), dtype=BF) for _ in "kv"], torch.zeros((9, 2), dtype=torch.int32)
    lens = torch.zeros(9, dtype=torch.int32)
    reaches_the_library(lambda: ssq.ssq_attention_decode(q[:, None], *pools, table, lens, 32))
    two = torch.zeros((2, 9, 64), dtype=BF).transpose(0, 1)             # two heads so laid out are not
    with pytest.raises(ValueError, match="contiguous"):
        ssq.ssq_attention_prompt(two, k, k, starts)
    with pytest.raises(ValueError, match="contiguous"):
        ssq.ssq_attention_decode(two[:, None], *pools, table, lens, 32)
