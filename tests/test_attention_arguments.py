"""More host-only checks of the attention part of the C ABI: arguments that would race or that no launch
can hold are refused before any HIP call."""
import pytest

from tests.test_attention_host import EINVAL, TABLES, call, off

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
