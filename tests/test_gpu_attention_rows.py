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


# Hidden keys and values of any bits: those that are no numbers, and the largest that are
BAD = [float("nan"), float("inf"), -float("inf"), 3e38]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("i", range(len(PROMPTS)))
def test_prompt_hidden_keys_of_any_bits_change_none(i, bad, dtype):
    lens, heads, p = PROMPTS[i]
    q, k, v = prompt_inputs(lens, heads, dtype, 310 + i)
    starts = ints(A.starts_of(lens))
    out = ssq.ssq_attention_prompt(sharp(q, 2.0), k, v, starts)
    for step in (1, 3):
        k2, v2 = k.clone(), v.clone()
        k2[p::step, :, ::3] = bad
        v2[p::step, :, 1::2] = bad
        check_bits(ssq.ssq_attention_prompt(sharp(q, 2.0), k2, v2, starts)[:p], out[:p], f"{lens} {heads} {bad} {step}")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("prefix", [0, 64, 100])
def test_decode_hidden_keys_of_any_bits_change_none(prefix, bad, dtype):
    """A late draft of one request, what another holds behind the prefix, and what no request holds; requests that
    end inside the prefix see less of it than others."""
    fresh, page, heads = 5, 16, (16, 2, 128)
    lens = [130, 97, 200] + [101 + i for i in range(20)]
    q, k, v, table, _ = cache_inputs(lens, fresh, prefix, page, heads, dtype, 330)
    out = run_decode(sharp(q, 2.0), k, v, table, lens, prefix)
    k2, v2 = k.clone(), v.clone()
    e, t = int(table[0, 128 // page]), 128 % page           # request 0: the fourth draft of five
    k2[e, :, t, ::3], v2[e, :, t, 1::2] = bad, bad
    for r, n in enumerate(lens):                            # past every request's end
        at = n % page
        if at:
            k2[int(table[r, n // page]), :, at:], v2[int(table[r, n // page]), :, at:] = bad, bad
    got = run_decode(sharp(q, 2.0), k2, v2, table, lens, prefix)
    check_bits(got[1:], out[1:], f"{bad}")
    check_bits(got[0, :3], out[0, :3], f"{bad} drafts")
    short = [60, 97] + lens[2:]
    if prefix:                                              # the prefix's later keys, which request 0 does not see
        first = run_decode(sharp(q, 2.0), k, v, table, short, prefix)
        for t in range(60, prefix):
            k2[int(table[0, t // page]), :, t % page, ::3] = bad
            v2[int(table[0, t // page]), :, t % page, 1::2] = bad
        check_bits(run_decode(sharp(q, 2.0), k2, v2, table, short, prefix)[0], first[0], f"{bad} short")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("lens,heads", [([150, 60], (8, 2, 64)), ([400], (4, 1, 128))])
def test_prompt_values_that_are_no_numbers_reach_exactly_the_rows_that_see_them(lens, heads, dtype):
    q, k, v = prompt_inputs(lens, heads, dtype, 350)
    starts, (hq, hk, d) = ints(A.starts_of(lens)), heads
    out = ssq.ssq_attention_prompt(q, k, v, starts)
    v2 = v.clone()
    v2[37, 0, 5], v2[100, 0, 6], v2[70, 0, 5] = float("inf"), float("nan"), -float("inf")
    got = ssq.ssq_attention_prompt(q, k, v2, starts).float()
    end, g = lens[0], hq // hk
    assert (got[37:70, :g, 5] == float("inf")).all() and torch.isnan(got[70:end, :g, 5]).all() and torch.isnan(got[100:end, :g, 6]).all()
    want = out.float()
    for a, c in ((37, 5), (100, 6)):
        got[a:end, :g, c] = want[a:end, :g, c] = 0
    check_bits(got, want, "the others")


# --- scores of minus infinity -------------------------------------------------------------------


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("lens,heads", [([5], (4, 2, 64)), ([150, 60], (32, 8, 128)), ([400], (4, 1, 128)), ([130, 2], (8, 8, 64))])
def test_prompt_rows_whose_scores_are_all_minus_infinity_are_nan(lens, heads, dtype):
    """Softmax over scores of -inf alone has no value; beside any finite score their weight is zero."""
    q, k, v = prompt_inputs(lens, heads, dtype, 400)
    q[..., 0] = 1 + q[..., 0].abs()
    starts = ints(A.starts_of(lens))
    first = min(lens[0] - 1, 67)
    k[:first, :, 0] = -float("inf")                          # every key of the first sequence before `first`
    out = ssq.ssq_attention_prompt(q, k, v, starts)
    assert torch.isnan(out[:first]).all()
    a, b = first, lens[0]
    A.check(out[a:b], *A.prompt_reference(q[a:b], k[a:b], v[a:b], [b - a]), "rows that see finite scores too")
    if len(lens) > 1:
        A.check(out[b:], *A.prompt_reference(q[b:], k[b:], v[b:], lens[1:]), "the other sequence")
    k[..., 0] = -float("inf")
    assert torch.isnan(ssq.ssq_attention_prompt(q, k, v, starts)).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("prefix", [0, 64, 90])
@pytest.mark.parametrize("n", [1, 3, 40])
def test_decode_rows_whose_scores_are_all_minus_infinity_are_nan(n, prefix, dtype):
    heads, page, fresh = (8, 2, 128), 16, 2
    lens = [(1900, 131, 92)[r % 3] + r for r in range(n)]
    q, k, v, table, _ = cache_inputs(lens, fresh, prefix, page, heads, dtype, 420 + n)
    q[..., 0] = 1 + q[..., 0].abs()
    bad = k.clone()
    bad[..., 0] = -float("inf")
    for ws in (None, torch.empty(0, dtype=torch.uint8, device="cuda")):
        assert torch.isnan(run_decode(q, bad, v, table, lens, prefix, workspace=ws)).all()
        # nothing seen is still nothing: no tokens, a token before the first, pages that are absent
        assert not run_decode(q, bad, v, table, [0] * n, prefix, max_len=max(lens), workspace=ws).any()
        one = run_decode(q, bad, v, table, [1] * n, prefix, max_len=max(lens), workspace=ws)
        assert not one[:, 0].any() and torch.isnan(one[:, 1]).all()
        assert not run_decode(q, bad, v, torch.full_like(table, -1), lens, prefix, workspace=ws).any()
    # the first page is absent and the rest -inf; then only the last key of every request is finite
    some = table.clone()
    some[:, 0] = -1
    assert torch.isnan(run_decode(q, bad, v, some, lens, prefix)).all()
    for r, m in enumerate(lens):
        bad[int(table[r, (m - 1) // page]), :, (m - 1) % page] = k[int(table[r, (m - 1) // page]), :, (m - 1) % page]
    for ws in (None, torch.empty(0, dtype=torch.uint8, device="cuda")):
        out = run_decode(q, bad, v, table, lens, prefix, workspace=ws)
        assert torch.isnan(out[:, 0]).all()
        for r, m in enumerate(lens):
            want = v[int(table[r, (m - 1) // page]), :, (m - 1) % page].repeat_interleave(4, 0)
            if dtype == BF:                                 # w v / w, to within binary32
                check_bits(out[r, 1], want, f"the value of the one finite key, request {r}")
            assert ((out[r, 1] - want).abs() <= 2.0 ** -20 * want.abs()).all()
