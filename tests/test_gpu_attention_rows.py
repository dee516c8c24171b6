"""A row of attention is a function of what it sees: its query, and the keys and values up to its own.
Whatever else shares its tile (later tokens, other requests, other heads) changes no bit of it."""
import pytest
import torch

from paper_2607_08779_amd import ssq
from tests import attention_common as A
from tests.test_gpu_attention import BF, F32, cache_inputs, gen, ints, prompt_inputs, run_decode

pytestmark = pytest.mark.gpu


def check_bits(a, b, tag):
    i = torch.int16 if a.dtype == BF else torch.int32
    off = int((a.contiguous().view(i) != b.contiguous().view(i)).sum())
    assert off == 0, f"{tag}: {off} of {a.numel()} differ"


def sharp(q, factor):
    """Scores that spread over more than the reference's slack, so that it moves, and by less than it too."""
    return (q.float() * factor).to(q.dtype)


# bf16: the kernel of 128 rows, then that of 32 (few rows, long sequences)
PROMPTS = [([180, 90], (32, 8, 128), 101), ([150, 0, 70], (8, 8, 64), 97), ([700], (4, 1, 128), 390), ([430], (4, 2, 64), 200)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("factor", [1.0, 3.0, 10.0])
@pytest.mark.parametrize("i", range(len(PROMPTS)))
def test_prompt_row_does_not_depend_on_later_tokens(i, factor, dtype):
    lens, heads, p = PROMPTS[i]
    q, k, v = prompt_inputs(lens, heads, dtype, 200 + i)
    q, starts = sharp(q, factor), ints(A.starts_of(lens))
    out = ssq.ssq_attention_prompt(q, k, v, starts)
    for times in (0.0, 1.0, 7.0):
        q2, k2, v2 = (x.clone() for x in (q, k, v))
        other = prompt_inputs(lens, heads, dtype, 300 + i)
        for x, y in zip((q2, k2, v2), other):
            x[p:] = (y[p:].float() * times).to(dtype)
        again = ssq.ssq_attention_prompt(q2, k2, v2, starts)
        check_bits(again[:p], out[:p], f"{lens} {heads} {times}")


DECODES = [
    # lens, fresh, prefix, page, heads: nothing shared, a few rows behind a prefix, many
    ([300, 40, 33, 500], 1, 0, 16, (32, 8, 128)),
    ([300, 290, 310], 2, 257, 16, (8, 2, 128)),
    ([330 + i for i in range(40)], 1, 320, 64, (8, 2, 64)),
    ([700 + 3 * i for i in range(21)], 3, 640, 32, (8, 1, 128)),
]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("factor", [1.0, 3.0, 10.0])
@pytest.mark.parametrize("i", range(len(DECODES)))
def test_decode_request_does_not_depend_on_the_others(i, factor, dtype):
    lens, fresh, prefix, page, heads = DECODES[i]
    q, k, v, table, lens = cache_inputs(lens, fresh, prefix, page, heads, dtype, 220 + i)
    q = sharp(q, factor)
    out = run_decode(q, k, v, table, lens, prefix)
    for r in (0, len(lens) // 2):
        for times in (0.0, 1.0, 7.0):
            q2 = sharp(A.model_like(gen(240 + i), q.shape, dtype), times)
            q2[r] = q[r]
            again = run_decode(q2, k, v, table, lens, prefix)
            check_bits(again[r], out[r], f"{DECODES[i]} request {r} times {times}")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("prefix", [0, 64])
def test_decode_draft_does_not_depend_on_later_ones(prefix, dtype):
    fresh, page, heads = 5, 16, (16, 2, 128)
    q, k, v, table, lens = cache_inputs([130, 97, 200], fresh, prefix, page, heads, dtype, 260)
    q = sharp(q, 4.0)
    out = run_decode(q, k, v, table, lens, prefix)
    for times in (0.0, 1.0, 7.0):
        q2, k2, v2 = (x.clone() for x in (q, k, v))
        for r, n in enumerate(lens):
            for t in (n - 2, n - 1):                        # the last two of five
                e = int(table[r, t // page])
                k2[e, :, t % page] = sharp(A.model_like(gen(270 + t), (heads[1], heads[2]), dtype), times)
                v2[e, :, t % page] = sharp(A.model_like(gen(280 + t), (heads[1], heads[2]), dtype), times)
        q2[:, 3:] = sharp(A.model_like(gen(290), (3, 2, heads[0], heads[2]), dtype), times)
        again = run_decode(q2, k2, v2, table, lens, prefix)
        check_bits(again[:, :3], out[:, :3], f"times {times}")
