"""How the attention operators may be called: buffers, layouts and sizes."""
import pytest
import torch

from paper_2607_08779_amd import ssq
from tests import attention_common as A
from tests.test_gpu_attention import ints

pytestmark = pytest.mark.gpu


def test_page_tables_lengths_of_one_step_are_held_by_the_next():
    """A serving loop in two sets of buffers, of more tokens than a workgroup takes; in one set it is refused."""
    n, page, width = 1500, 16, 6
    held, taken, table = [7 * i % 40 for i in range(n)], 0, [[-1] * width for _ in range(n)]
    free = list(range(n * width))
    dev, dev_free = ints(table), ints(free)
    sets = [[torch.empty(k, dtype=torch.int32, device="cuda") for k in (n + 1, n, n, n, 1)] for _ in range(2)]
    sets[1][1].copy_(ints(held))
    sets[1][4].zero_()
    for step in range(4):
        before, now = sets[(step + 1) % 2], sets[step % 2]
        got = ssq.ssq_page_tables(before[1], ints([1] * n), dev_free, dev, page, n, taken=before[4], out=now)
        want = A.tables_reference(held, [1] * n, free, taken, page, table, n)
        assert [x.tolist() if j != 4 else x.item() for j, x in enumerate(got)] == list(want)
        held, taken, table = want[1], want[4], want[5]
        for bad in ([*now[:1], before[1], *now[2:]], [before[1].new_empty(n + 1), now[1], now[1], *now[3:]]):
            with pytest.raises(ssq.SSQError):
                ssq.ssq_page_tables(before[1], ints([1] * n), dev_free, dev, page, n, taken=before[4], out=bad)


def test_decode_of_as_many_requests_as_a_launch_holds():
    """2^20 requests of 15 heads, a workgroup each: those of no token give zeros, of one token its value."""
    n, heads, d, page = 1 << 20, 15, 64, 16
    gen = torch.Generator(device="cuda").manual_seed(500)
    k, v = (torch.randn((4, heads, page, d), generator=gen, device="cuda").bfloat16() for _ in "kv")
    q = torch.randn((n, 1, heads, d), generator=gen, device="cuda", dtype=torch.bfloat16)
    request = torch.arange(n, device="cuda", dtype=torch.int32)
    lens, table = request % 2, (request % 4)[:, None].contiguous()
    out = ssq.ssq_attention_decode(q, k, v, table, lens, page)
    assert not out[::2].any()
    for r in (1, 3):
        assert (out[r::4, 0] == v[r, :, 0]).all()


def test_one_head_of_a_tensor_of_heads_first():
    """[heads, tokens, dim] transposed: with one head a token's row, whatever the stride between heads."""
    gen = torch.Generator(device="cuda").manual_seed(510)
    q, k, v = (torch.randn((1, 60, 64), generator=gen, device="cuda").bfloat16()[:, 3:53].transpose(0, 1) for _ in "qkv")
    starts = ints([0, 30, 50])
    A.check(ssq.ssq_attention_prompt(q, k, v, starts), *A.prompt_reference(q, k, v, [30, 20]), "one head")
    pos, rope = torch.arange(50, device="cuda", dtype=torch.int32), torch.randn((50, 64), generator=gen, device="cuda")
    for a, b in zip(ssq.ssq_qk_norm_rope(q, k, pos, rope), ssq.ssq_qk_norm_rope(q.clone().contiguous(), k.clone().contiguous(), pos, rope)):
        assert torch.equal(a, b)
    pools = [torch.randn((4, 1, 16, 64), generator=gen, device="cuda").bfloat16() for _ in "kv"]
    table, lens = ints([[r % 4, 3] for r in range(50)]), [r % 33 for r in range(50)]
    out = ssq.ssq_attention_decode(q[:, None], *pools, table, ints(lens), 32)
    A.check(out, *A.decode_reference(q[:, None], *pools, table.cpu(), lens, 32, 0), "one head, decoding")
