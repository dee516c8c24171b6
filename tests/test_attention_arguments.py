"""More host-only checks of the attention part of the C ABI: arguments that would race or that no launch
can hold are refused before any HIP call."""
import pytest

from paper_2607_08779_amd import ssq
from tests.test_attention_host import DECODE, EALIGN, EINVAL, PROMPT, ROPE, TABLES, call, off

# Arrays of the page tables' call 256 KB apart, none of them over another: 2 requests, 4 free pages, rows
# of 3 pages, 5 tokens
APART = {name: off(i << 18) for i, name in enumerate(
    ("held", "added", "free_pages", "taken", "table", "starts", "lens", "positions", "slots", "taken_after"))}
COUNT = dict(held=2, added=2, free_pages=4, taken=1, table=6, starts=3, lens=2, positions=5, slots=5, taken_after=1)
WRITTEN = ("table", "starts", "lens", "positions", "slots", "taken_after")


@pytest.mark.parametrize("written", WRITTEN)
@pytest.mark.parametrize("other", list(COUNT))
def test_page_tables_refuses_outputs_over_other_arrays(written, other):
    """Workgroups read the lengths, the free list and the rows while others write: an output over an input
    (the lengths of one step as the next one's, in place) or over another output is a race."""
    if other == written:
        return
    start = APART[other].value
    for first in {start, start + 4 * (COUNT[other] - 1), start - 4 * (COUNT[written] - 1)}:    # the whole, its last element, its first
        assert call("ssq_page_tables", TABLES, {**APART, written: type(APART[other])(first)}) == EINVAL, (written, other, first - start)


# --- sizes: a launch holds fewer than 2^24 workgroups of 256 threads ---------------------------

@pytest.mark.parametrize("name,size", [("ssq_qk_norm_rope", 2), ("ssq_qk_norm_rope_f32", 4)])
@pytest.mark.parametrize("dim", [64, 128])
def test_norm_rope_refuses_what_no_launch_holds(name, size, dim):
    """32 bytes a thread: 127 GiB of heads are the last whole GiB that fit, and the next head is refused."""
    heads = (127 << 30) // (size * dim)
    given = dict(q_heads=1, kv_heads=1, head_dim=dim, q_stride=dim, k_stride=dim, v_stride=dim, q_out_stride=dim, k_out_stride=dim)
    assert call(name, ROPE, {**given, "tokens": heads // 3 + 1}) == EINVAL
    assert call(name, ROPE, {**given, "tokens": heads // 3, "q": off(8)}) == EALIGN          # past the sizes


@pytest.mark.parametrize("name,rows", [("ssq_attention_prompt", 128), ("ssq_attention_prompt_f32", 32)])
def test_prompt_refuses_what_no_launch_holds(name, rows):
    """ceil(tokens * group / rows) + requests workgroups a key/value head."""
    wide = dict(k_stride=1 << 11, v_stride=1 << 11, q_stride=1 << 11, out_stride=1 << 11, q=off(8))
    at = dict(requests=1 << 20, q_heads=16, kv_heads=16)
    assert call(name, PROMPT, {**wide, **at, "tokens": 1}) == EINVAL                         # 2^24 of them for the requests alone
    assert call(name, PROMPT, {**wide, **at, "requests": (1 << 20) - 2, "tokens": 1}) == EALIGN
    one = dict(requests=1, q_heads=16, kv_heads=1)
    most = (rows * (1 << 24) - 1 - rows * 2) // 16
    assert call(name, PROMPT, {**wide, **one, "tokens": most + 1}) == EINVAL
    assert call(name, PROMPT, {**wide, **one, "tokens": most}) == EALIGN


def test_decode_refuses_what_no_launch_holds():
    """ceil(fresh * group / 32) workgroups a request and key/value head."""
    for name in ("ssq_attention_decode", "ssq_attention_decode_f32"):
        wide = dict(q_stride=1 << 11, out_stride=1 << 11, q=off(8), fresh=1)
        assert call(name, DECODE, {**wide, "requests": 1 << 20, "q_heads": 16, "kv_heads": 16}) == EINVAL
        assert call(name, DECODE, {**wide, "requests": 1 << 20, "q_heads": 15, "kv_heads": 15}) == EALIGN
        assert call(name, DECODE, {**wide, "requests": 1, "fresh": (1 << 25) - 2, "q_heads": 16, "kv_heads": 1}) == EINVAL
        assert call(name, DECODE, {**wide, "requests": 1, "fresh": (1 << 25) - 3, "q_heads": 16, "kv_heads": 1}) == EALIGN


def test_decode_splits_nothing_that_no_launch_holds():
    """A wavefront joins a row, so that parts are for fewer than 2^26 rows."""
    size = ssq.ssq_attention_decode_workspace_size
    assert size(1 << 20, 1, 63, 7, 64, 4096, 2048) > 0
    assert size(1 << 20, 1, 64, 8, 64, 4096, 2048) == 0
    assert size(1 << 20, 1, 16, 16, 64, 4096, 2048) == 0                                     # refused
