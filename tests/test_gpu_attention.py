"""The attention operators on the GPU against the same in 64 bits (tests/attention_common.py)."""
import pytest
import torch

from paper_2607_08779_amd import ssq
from tests import attention_common as A

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


# --- prompts ------------------------------------------------------------------------------------

def prompt_inputs(lens, heads, dtype, seed, fused=False, pad=0):
    hq, hk, d = heads
    g = gen(seed)
    t = sum(lens) + pad
    q, k, v = (A.model_like(g, (t, h, d), dtype) for h in (hq, hk, hk))
    if fused:
        q, k, v = torch.cat((q, k, v), 1).split((hq, hk, hk), 1)
    return q, k, v


PROMPTS = [
    ([1], (4, 4, 64)), ([2, 1], (32, 8, 128)), ([0, 1, 0, 5, 0], (8, 2, 64)), ([31, 32, 33], (32, 8, 128)),
    ([63, 64, 65, 1], (4, 1, 128)), ([127, 128, 129], (5, 5, 128)), ([200, 3, 77], (14, 2, 64)),
    ([513], (40, 8, 128)), ([150, 0, 260], (2, 2, 64)), ([90], (130, 1, 64)), ([17, 9], (64, 1, 128)),
    ([3] * 70, (4, 2, 64)),
]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("i", range(len(PROMPTS)))
def test_prompt(i, dtype):
    lens, heads = PROMPTS[i]
    pad = (0, 3, 40)[i % 3]
    q, k, v = prompt_inputs(lens, heads, dtype, i, fused=i % 2 == 1, pad=pad)
    out = ssq.ssq_attention_prompt(q, k, v, ints(A.starts_of(lens)))
    ref, size, eps = A.prompt_reference(q, k, v, lens)
    A.check(out, ref, size, eps, f"{lens} {heads} {dtype}")
    assert not out[sum(lens):].any()


def test_prompt_of_no_sequences_and_no_tokens():
    q, k, v = prompt_inputs([], (8, 2, 64), BF, 1, pad=300)
    assert not ssq.ssq_attention_prompt(q, k, v, ints([0])).any()
    assert ssq.ssq_attention_prompt(q[:0], k[:0], v[:0], ints([0, 0])).shape == (0, 8, 64)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_prompt_starts_outside_the_tokens_are_clamped(dtype):
    q, k, v = prompt_inputs([50], (8, 2, 64), dtype, 2)
    out = ssq.ssq_attention_prompt(q, k, v, ints([0, 20, 10, 2 ** 31 - 1]))   # 20, none, 10..50
    want = torch.zeros_like(out)
    A.check(out[:10], *[x[:10] for x in A.prompt_reference(q, k, v, [20, 30])], "before the overlap")
    A.check(out[20:], *[x[20:] for x in A.prompt_reference(torch.cat((q[:10], q[10:])), k, v, [10, 40])], "the last sequence")
    assert torch.isfinite(out).all() and want.shape == out.shape


@pytest.mark.parametrize("factor", [0.0, 30.0, 1e4])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_prompt_flat_and_sharp_scores(factor, dtype):
    lens, heads = [140, 71], (8, 2, 128)
    q, k, v = prompt_inputs(lens, heads, dtype, 3)
    q = (q.float() * factor).to(dtype)
    out = ssq.ssq_attention_prompt(q, k, v, ints(A.starts_of(lens)))
    A.check(out, *A.prompt_reference(q, k, v, lens), f"factor {factor}")


def test_prompt_rising_scores_move_the_reference():
    """Each key outscores all before it by far: the running reference moves at every tile."""
    n, d = 400, 64
    g = gen(4)
    v = A.model_like(g, (n, 1, d), BF)
    q = torch.ones((n, 2, d), device="cuda", dtype=BF)
    k = (torch.arange(n, device="cuda", dtype=F32) * 0.25)[:, None, None].expand(n, 1, d).to(BF).contiguous()
    out = ssq.ssq_attention_prompt(q, k, v, ints([0, n]))
    A.check(out, *A.prompt_reference(q, k, v, [n]), "rising")
    out = ssq.ssq_attention_prompt(q, -k, v, ints([0, n]))
    A.check(out, *A.prompt_reference(q, -k, v, [n]), "falling")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("heads", [(8, 2, 128), (6, 6, 64)])
def test_prompt_hidden_keys_have_no_influence(dtype, bad, heads):
    """Infinities and NaN in later tokens and in other sequences."""
    lens = [70, 130, 45]
    q, k, v = prompt_inputs(lens, heads, dtype, 5, pad=9)
    ref, size, eps = A.prompt_reference(q, k, v, lens)
    k, v = k.clone(), v.clone()
    at = [41, 70 + 64, 70 + 101, 200, 246]
    for t in at:
        k[t, :, ::3] = bad
        v[t, :, 1::2] = bad
    out = ssq.ssq_attention_prompt(q, k, v, ints(A.starts_of(lens)))
    seen = [range(0, 41), range(70, 134), ]
    for rows in seen:
        A.check(out[rows[0]:rows[-1] + 1], *(x[rows[0]:rows[-1] + 1] for x in (ref, size, eps)), f"{bad} {rows}")
    assert out[70:134].isfinite().all() and out[200].isfinite().all().item() is False
    k2, v2 = k.clone(), v.clone()
    k2[200, :, ::3], v2[200, :, 1::2] = 1, 1
    assert not out[246:].any()                                    # padding


def test_prompt_values_that_are_infinite_reach_the_rows_that_see_them():
    lens = [100]
    q, k, v = prompt_inputs(lens, (4, 2, 64), BF, 6)
    v[37, 0, 5] = float("inf")
    v[60, 1, 7] = float("nan")
    out = ssq.ssq_attention_prompt(q, k, v, ints([0, 100])).float()
    assert torch.isinf(out[37:, :2, 5]).all() and torch.isfinite(out[:37]).all()
    assert torch.isnan(out[60:, 2:, 7]).all() and torch.isfinite(out[:60, 2:]).all()
    out[37:, :2, 5] = 0
    out[60:, 2:, 7] = 0
    assert torch.isfinite(out).all()


def test_prompt_long_rows():
    """2500 tokens: sampled rows, and the two halves as sequences of their own."""
    for lens in ([2500], [1300, 1200]):
        q, k, v = prompt_inputs(lens, (32, 8, 128), BF, 7)
        out = ssq.ssq_attention_prompt(q, k, v, ints(A.starts_of(lens)))
        a = 0
        for n in lens:
            rows = torch.tensor([0, 1, 63, 64, 500, n - 2, n - 1])
            for h in (0, 13, 31):
                ref, size, eps = A.attend(q[a + rows, h], k[a:a + n, h // 4], v[a:a + n, h // 4], rows, 128 ** -0.5)
                A.check(out[a + rows, h], ref, size, eps, f"{lens} head {h}")
            a += n


def test_prompt_writes_only_its_rows():
    lens, (hq, hk, d) = [37, 60], (8, 2, 64)
    q, k, v = prompt_inputs(lens, (hq, hk, d), BF, 8)
    wide = torch.full((97, hq + 3, d), 7.0, dtype=BF, device="cuda")
    out = ssq.ssq_attention_prompt(q, k, v, ints(A.starts_of(lens)), out=wide[:, 1:hq + 1])
    A.check(out, *A.prompt_reference(q, k, v, lens), "strided out")
    assert (wide[:, 0] == 7).all() and (wide[:, hq + 1:] == 7).all()


# Few rows and long sequences: in bf16 the kernel of 32 rows a workgroup, its neighbours around the rule
FEW = [
    ([97], (4, 4, 64)), ([430], (4, 1, 128)), ([129, 0, 300], (8, 2, 64)), ([321], (8, 2, 128)),
    ([800], (6, 1, 128)), ([1100, 3], (14, 2, 64)), ([333, 340], (2, 2, 128)), ([95], (4, 4, 64)), ([319], (8, 2, 128)),
]


@pytest.mark.parametrize("i", range(len(FEW)))
def test_prompt_few_rows(i):
    lens, heads = FEW[i]
    q, k, v = prompt_inputs(lens, heads, BF, 80 + i, fused=i % 2 == 0, pad=(0, 35)[i % 2])
    wide = torch.full((len(q), heads[0] + 2, heads[2]), 7.0, dtype=BF, device="cuda")
    out = ssq.ssq_attention_prompt(q, k, v, ints(A.starts_of(lens)), out=wide[:, 1:heads[0] + 1])
    ref, size, eps = A.prompt_reference(q, k, v, lens)
    A.check(out, ref, size, eps, f"{lens} {heads}")
    assert not out[sum(lens):].any() and (wide[:, 0] == 7).all() and (wide[:, -1] == 7).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("heads", [(8, 2, 128), (6, 6, 64)])
def test_prompt_few_rows_hidden_keys_have_no_influence(bad, heads):
    lens = [400, 350]
    q, k, v = prompt_inputs(lens, heads, BF, 90, pad=11)
    ref, size, eps = A.prompt_reference(q, k, v, lens)
    k, v = k.clone(), v.clone()
    for t in (37, 161, 400 + 77, 755):
        k[t, :, ::3] = bad
        v[t, :, 1::2] = bad
    out = ssq.ssq_attention_prompt(q, k, v, ints(A.starts_of(lens)))
    for a, b in ((0, 37), (400, 477)):
        A.check(out[a:b], ref[a:b], size[a:b], eps[a:b], f"{bad} {a}")
    assert not out[477:750].isfinite().all() and not out[750:].any()


def test_prompt_scale_and_repeat():
    lens = [90, 33]
    q, k, v = prompt_inputs(lens, (8, 2, 64), BF, 9)
    out = ssq.ssq_attention_prompt(q, k, v, ints(A.starts_of(lens)), scale=0.3)
    A.check(out, *A.prompt_reference(q, k, v, lens, scale=0.3), "scale")
    again = ssq.ssq_attention_prompt(q, k, v, ints(A.starts_of(lens)), scale=0.3)
    assert torch.equal(out, again)


def test_rows_of_one_key_give_its_value():
    """The weights' rounding cancels in a row of one key: w v / w, to within binary32, is v in bf16."""
    q, k, v = prompt_inputs([1] * 200, (8, 2, 128), BF, 95)
    out = ssq.ssq_attention_prompt(q * 3, k, v, torch.arange(201, device="cuda", dtype=torch.int32))
    assert torch.equal(out, v.repeat_interleave(4, 1))
    q, kp, vp, table, lens = cache_inputs([1] * 50, 1, 0, 16, (8, 2, 64), BF, 96)
    out = run_decode(q * 3, kp, vp, table, lens, 0)
    want = vp[table[:, 0].long().cuda(), :, 0]
    assert torch.equal(out[:, 0], want.repeat_interleave(4, 1))


# --- decoding -----------------------------------------------------------------------------------

def cache_inputs(lens, fresh, prefix, page, heads, dtype, seed, poison=None, spare=3, extra=0):
    """Caches whose every slot that no request should see holds `poison`."""
    hq, hk, d = heads
    g = gen(seed)
    n = len(lens)
    shared = prefix // page
    need = [max(A.pages_for(x, page) - shared, 0) for x in lens]
    pages = shared + sum(need) + spare
    ids = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    width = max(1, shared + max(need)) + extra
    table = torch.full((n, width), -7, dtype=torch.int32)
    at = shared
    for r in range(n):
        table[r, :shared] = ids[:shared]
        table[r, shared:shared + need[r]] = ids[at:at + need[r]]
        at += need[r]
    k, v = (torch.full((pages, hk, page, d), 0.0 if poison is None else poison, dtype=dtype, device="cuda") for _ in "kv")
    top = max([prefix] + lens)
    base_k, base_v = (A.model_like(g, (max(top, 1), hk, d), dtype) for _ in "kv")
    for r in range(n):
        mine = A.model_like(g, (max(top, 1), hk, d), dtype), A.model_like(g, (max(top, 1), hk, d), dtype)
        for t0 in range(0, lens[r], page):
            e, m = int(table[r, t0 // page]), min(page, lens[r] - t0)
            for pool, own, base in ((k, mine[0], base_k), (v, mine[1], base_v)):
                rows = torch.where((torch.arange(t0, t0 + m, device="cuda") < prefix)[:, None, None], base[t0:t0 + m], own[t0:t0 + m])
                pool[e, :, :m] = rows.transpose(0, 1)
                if poison is not None and r > 0 and t0 < prefix < t0 + page:
                    pool[e, :, :prefix - t0] = poison        # read from request 0's page only
    q = A.model_like(g, (n, fresh, hq, d), dtype)
    return q, k, v, table, lens


def run_decode(q, k, v, table, lens, prefix, max_len=None, **more):
    return ssq.ssq_attention_decode(q, k, v, table.cuda(), ints(lens), max(lens) if max_len is None else max_len, prefix=prefix, **more)


DECODES = [
    # lens, fresh, prefix, page, heads
    ([1], 1, 0, 16, (4, 4, 64)),
    ([33, 1, 64, 500], 1, 0, 16, (32, 8, 128)),
    ([0, 5, 0], 1, 0, 16, (8, 2, 64)),
    ([700], 1, 0, 64, (40, 8, 128)),
    ([100, 130, 101], 1, 100, 16, (32, 8, 128)),           # narrow sharing, prefix inside a page
    ([96, 100, 97, 160, 96], 1, 96, 32, (14, 2, 64)),
    ([300, 40, 333, 0], 1, 297, 64, (8, 1, 128)),          # shorter than the prefix
    ([270 + i for i in range(20)], 1, 257, 16, (8, 2, 128)),      # wide sharing
    ([70 + 9 * i for i in range(40)], 2, 64, 16, (16, 4, 64)),
    ([10, 3, 1, 0, 25], 4, 0, 16, (8, 2, 128)),            # tokens before the first key
    ([150, 170], 9, 120, 32, (32, 4, 64)),                 # more rows than a tile
    ([600, 650, 700], 3, 512, 128, (6, 6, 128)),
    ([50, 60], 1, 40, 1024, (130, 1, 64)),
    ([1100, 1030], 1, 1024, 16, (8, 8, 64)),
]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("i", range(len(DECODES)))
def test_decode(i, dtype):
    lens, fresh, prefix, page, heads = DECODES[i]
    q, k, v, table, lens = cache_inputs(lens, fresh, prefix, page, heads, dtype, 20 + i, poison=float("nan"))
    ref, size, eps = A.decode_reference(q, k, v, table, lens, max(lens), prefix)
    for name, more in (("workspace", {}), ("none", {"workspace": torch.empty(0, dtype=torch.uint8, device="cuda")})):
        print(DECODES[i], dtype, name, flush=True)
        out = run_decode(q, k, v, table, lens, prefix, **more)
        A.check(out, ref, size, eps, f"{DECODES[i]} {dtype} {name}")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("prefix", [0, 90])
def test_decode_absent_pages(dtype, prefix):
    lens = [200, 230, 190]
    q, k, v, table, lens = cache_inputs(lens, 1, prefix, 16, (8, 2, 64), dtype, 40, poison=float("inf"))
    table[1, 9], table[2, 6], table[2, 11] = -1, k.shape[0], 2 ** 31 - 1
    if prefix:
        table[:, 2] = -5
    ref, size, eps = A.decode_reference(q, k, v, table, lens, 230, prefix)
    for ws in (None, torch.empty(0, dtype=torch.uint8, device="cuda")):
        A.check(run_decode(q, k, v, table, lens, prefix, workspace=ws), ref, size, eps, f"absent {prefix}")


def test_decode_all_pages_absent_or_no_pages():
    q, k, v, table, lens = cache_inputs([40, 50], 1, 0, 16, (8, 2, 64), BF, 41)
    assert not run_decode(q, k, v, torch.full_like(table, -1), lens, 0).any()
    assert not run_decode(q, k[:0], v[:0], table, lens, 0).any()
    assert not run_decode(q, k, v, table[:, :0].contiguous(), lens, 0).any()
    assert not run_decode(q, k, v, table, [0, -3], 0, max_len=50).any()
    assert not run_decode(q, k, v, table, lens, 0, max_len=0).any()
    assert run_decode(q[:0], k, v, table[:0], [], 0, max_len=5).shape == (0, 1, 8, 64)


def test_decode_lengths_are_bounded():
    lens = [500, 90]
    q, k, v, table, _ = cache_inputs(lens, 1, 0, 16, (8, 2, 64), BF, 42)
    for max_len, width in ((120, table.shape[1]), (500, 3), (2 ** 30, 4)):
        t = table[:, :width].contiguous()
        ref, size, eps = A.decode_reference(q, k, v, t, lens, max_len, 0)
        A.check(run_decode(q, k, v, t, lens, 0, max_len=max_len), ref, size, eps, f"{max_len} {width}")
    ref, size, eps = A.decode_reference(q, k, v, table, [500, 90], 500, 0)
    A.check(run_decode(q, k, v, table, lens, 0, max_len=100000), ref, size, eps, "a wide bound")


# Many rows behind a longer prefix: several row tiles and parts, their numbers not those of the chip
MANY = [
    ([900 + 7 * i for i in range(30)], 3, 890, 32, (9, 3, 128)),
    ([1300 + i for i in range(45)], 5, 1281, 64, (8, 1, 64)),
    ([640 + (37 * i) % 300 for i in range(21)], 1, 640, 16, (28, 7, 64)),
]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("prefix", [0, 70])
@pytest.mark.parametrize("n", [64, 65, 131])
def test_decode_requests_of_all_lengths(n, prefix, dtype):
    """More requests than places, so that they are taken longest first: empty, equal and long ones."""
    some = [0, 700, 33, 700, 1, 64, 699, 5, 128, 0, 300]
    lens = [0 if some[r % 11] == 0 else prefix + some[r % 11] - r % 3 * (some[r % 11] > 9) for r in range(n)]
    heads = (18, 9, 64)
    q, k, v, table, _ = cache_inputs(lens, 1, prefix, 64, heads, dtype, 120 + n, poison=float("nan"))
    ref, size, eps = A.decode_reference(q, k, v, table, lens, max(lens), prefix)
    A.check(run_decode(q, k, v, table, lens, prefix), ref, size, eps, f"{n} {prefix} {dtype}")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("i", range(len(MANY)))
def test_decode_many_rows_behind_a_prefix(i, dtype):
    lens, fresh, prefix, page, heads = MANY[i]
    q, k, v, table, lens = cache_inputs(lens, fresh, prefix, page, heads, dtype, 100 + i, poison=float("nan"))
    ref, size, eps = A.decode_reference(q, k, v, table, lens, max(lens), prefix)
    A.check(run_decode(q, k, v, table, lens, prefix), ref, size, eps, f"{heads} {dtype}")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_decode_later_drafts_have_no_influence(dtype, bad):
    lens, fresh, prefix = [130, 97, 64], 5, 60
    q, k, v, table, _ = cache_inputs(lens, fresh, prefix, 16, (8, 2, 128), dtype, 43)
    ref, size, eps = A.decode_reference(q, k, v, table, lens, 130, prefix)
    for r in range(3):
        t = lens[r] - 2                                     # the fourth of five
        k[table[r, t // 16], :, t % 16, ::2] = bad
        v[table[r, t // 16], :, t % 16, 1::2] = bad
    for ws in (None, torch.empty(0, dtype=torch.uint8, device="cuda")):
        out = run_decode(q, k, v, table, lens, prefix, workspace=ws)
        A.check(out[:, :3], ref[:, :3], size[:, :3], eps[:, :3], f"drafts {bad}")
        assert not out[:, 3:].isfinite().all()


def test_decode_reads_a_strided_query():
    lens = [60, 75, 80]
    q, k, v, table, _ = cache_inputs(lens, 1, 32, 16, (8, 2, 64), BF, 44)
    fused = torch.randn((3, 1, 12, 64), device="cuda").to(BF)
    fused[:, :, :8] = q
    ref, size, eps = A.decode_reference(q, k, v, table, lens, 80, 32)
    A.check(run_decode(fused[:, :, :8], k, v, table, lens, 32), ref, size, eps, "strided")


def test_decode_cache_past_32_bit_offsets():
    """Pages whose elements lie past 2^32 of a cache of 8.9 GB."""
    hk, d, page = 8, 128, 64
    pages = 2 ** 32 // (hk * d * page) + 300
    lens, prefix = [300, 261, 290], 256
    q, k, v, table, _ = cache_inputs(lens, 1, prefix, page, (32, hk, d), BF, 45)
    used = sorted({int(x) for r, n in zip(table, lens) for x in r[:A.pages_for(n, page)]})
    big_k, big_v = (torch.full((pages, hk, page, d), float("nan"), dtype=BF, device="cuda") for _ in "kv")
    moved = table.clone()
    for i, e in enumerate(used):
        big_k[pages - 1 - i * 7], big_v[pages - 1 - i * 7] = k[e], v[e]
        moved[table == e] = pages - 1 - i * 7
    ref, size, eps = A.decode_reference(q, k, v, table, lens, 300, prefix)
    A.check(run_decode(q, big_k, big_v, moved, lens, prefix), ref, size, eps, "far pages")
    del big_k, big_v
    torch.cuda.empty_cache()


def test_decode_long_cache_split():
    lens = [5000, 4097, 64]
    q, k, v, table, _ = cache_inputs(lens, 1, 0, 64, (8, 2, 128), BF, 46, poison=float("nan"))
    ref, size, eps = A.decode_reference(q, k, v, table, lens, 5000, 0)
    A.check(run_decode(q, k, v, table, lens, 0), ref, size, eps, "long")
    assert torch.equal(run_decode(q, k, v, table, lens, 0), run_decode(q, k, v, table, lens, 0))


# --- tables -------------------------------------------------------------------------------------

TABLES = [
    # held, added, page, free, taken, width, spare tokens
    ([0], [1], 16, 4, 0, 2, 0),
    ([15, 16, 17, 0, 31], [1, 1, 1, 1, 1], 16, 9, 2, 4, 3),
    ([0, 0, 5], [0, 0, 0], 16, 9, 0, 3, 2),
    ([100, 0, 64, 1], [300, 77, 64, 0], 64, 20, 1, 8, 0),
    ([100, 0, 64, 1], [300, 77, 64, 0], 32, 6, 1, 8, 5),          # too few free pages
    ([5, 40], [100, 9], 16, 30, 0, 3, 0),                          # rows too short
    ([-4, 3], [5, -2], 16, 30, 0, 3, 4),
    ([7], [5000], 16, 400, 0, 320, 1),
    ([3 * i % 50 for i in range(1500)], [i % 4 for i in range(1500)], 16, 3000, 5, 5, 100),
    ([0] * 300, [37] * 300, 1024, 300, 0, 1, 0),
    ([2 ** 31 - 2000], [100], 1024, 5, 0, 3, 0),
]


@pytest.mark.parametrize("i", range(len(TABLES)))
def test_page_tables(i):
    held, added, page, free_count, taken, width, spare = TABLES[i]
    n = len(held)
    ids = torch.randperm(5000, generator=torch.Generator().manual_seed(i)).tolist()
    table = [[ids[(r * width + j) % 5000] for j in range(width)] for r in range(n)]
    free = [5000 + x for x in ids[:free_count]]
    tokens = sum(max(a, 0) for a in added) + spare
    want = A.tables_reference(held, added, free, taken, page, table, tokens)
    dev = ints(table)
    for again in range(2):                                 # the same call again gives the same
        got = ssq.ssq_page_tables(ints(held), ints(added), ints(free), dev, page, tokens, taken=ints([taken]))
        assert [x.tolist() if j != 4 else x.item() for j, x in enumerate(got)] == list(want)
    assert got[5].data_ptr() == dev.data_ptr()


def test_page_tables_without_requests_and_with_short_outputs():
    e = ints([])
    starts, lens, pos, slots, taken, _ = ssq.ssq_page_tables(e, e, e, ints([]).view(0, 3), 16, 5)
    assert starts.tolist() == [0] and pos.tolist() == [0] * 5 and slots.tolist() == [-1] * 5 and taken.tolist() == [0]
    held, added, free = [0, 20], [40, 30], list(range(9))
    want = A.tables_reference(held, added, free, 0, 16, [[90] * 4] * 2, 50)     # 70 tokens, room for 50
    got = ssq.ssq_page_tables(ints(held), ints(added), ints(free), ints([[90] * 4] * 2), 16, 50)
    assert got[2].tolist() == want[2] and got[3].tolist() == want[3] and got[0].tolist() == [0, 40, 70]


# --- norm and rotation --------------------------------------------------------------------------

def rope_table(rows, d):
    angle = torch.arange(rows, device="cuda", dtype=torch.float64)[:, None] * 1e6 ** (-torch.arange(0, d, 2, device="cuda", dtype=torch.float64) / d)
    return torch.cat((angle.cos(), angle.sin()), 1).float()


def close(out, ref, size, tag):
    """A handful of binary32 operations on each element (its square sum over d elements, a
    reciprocal root, two products, a product and a sum): within 2^-18 of the terms' sizes, and
    half an ulp of bf16 where the output is that."""
    bound = size * 2.0 ** -18 + (ref.abs() * 2.0 ** -8 if out.dtype == BF else 0)
    bad = ~((out.double() - ref).abs() <= bound)
    assert not bad.any(), f"{tag}: {int(bad.sum())} of {bad.numel()} off"


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("tokens,heads,gain,fused,page", [
    (1, (32, 8, 128), True, False, 16), (7, (14, 2, 64), True, True, 32), (65, (5, 5, 128), False, True, 64),
    (3, (1, 1, 64), True, False, 1024), (300, (40, 8, 128), True, True, 16), (33, (8, 1, 64), False, False, 0),
])
def test_norm_rope(tokens, heads, gain, fused, page, dtype):
    hq, hk, d = heads
    q, k, v = prompt_inputs([tokens], heads, dtype, 60 + tokens, fused=fused)
    g = gen(61)
    gains = [(1 + 0.3 * torch.randn(d, generator=g, device="cuda")).to(dtype) if gain else None for _ in "qk"]
    table = rope_table(5000, d)
    pos = torch.randint(0, 5000, (tokens,), generator=g, device="cuda", dtype=torch.int32)
    more = {}
    if page:
        pages = A.pages_for(tokens, page) + 2
        before = torch.randn((2, pages, hk, page, d), generator=g, device="cuda").to(dtype)
        more = {"v": v, "k_pages": before[0].clone(), "v_pages": before[1].clone()}
        slots = torch.randperm(pages * page, generator=g, device="cuda")[:tokens].to(torch.int32)
        slots[tokens // 2] = -1 if tokens > 1 else slots[0]
        if tokens > 2:
            slots[0], slots[-1] = pages * page, 2 ** 31 - 1
        more["slots"] = slots
    qo, ko = ssq.ssq_qk_norm_rope(q, k, pos, table, q_gain=gains[0], k_gain=gains[1], eps=1e-5, **more)
    for x, y, w in ((q, qo, gains[0]), (k, ko, gains[1])):
        close(y, *A.rope_reference(x, w, table[pos.long()], 1e-5), f"{tokens} {heads} {dtype}")
    if page:
        for pool, rows, old in ((more["k_pages"], ko, before[0]), (more["v_pages"], v, before[1])):
            want = old.transpose(1, 2).reshape(-1, hk, d).clone()
            ok = (slots >= 0) & (slots < pages * page)
            want[slots[ok].long()] = rows[ok]
            assert torch.equal(pool, want.view(pages, page, hk, d).transpose(1, 2))


def test_norm_rope_in_place_and_cache_only():
    heads = (8, 2, 128)
    q, k, v = prompt_inputs([40], heads, BF, 70, fused=True)
    table, pos = rope_table(64, 128), torch.arange(40, device="cuda", dtype=torch.int32)
    gain = torch.full((128,), 1.25, device="cuda", dtype=BF)
    want = ssq.ssq_qk_norm_rope(q, k, pos, table, q_gain=gain)
    pools = [torch.zeros((3, 2, 16, 128), device="cuda", dtype=BF) for _ in "kv"]
    qq = torch.empty_like(want[0])
    ssq.ssq_qk_norm_rope(q, k, pos, table, q_gain=gain, v=v, slots=pos, k_pages=pools[0], v_pages=pools[1], out=(qq, None))
    assert torch.equal(qq, want[0])
    assert torch.equal(pools[0].transpose(1, 2).reshape(48, 2, 128)[:40], want[1])
    assert torch.equal(pools[1].transpose(1, 2).reshape(48, 2, 128)[:40], v)
    kept = v.clone()
    got = ssq.ssq_qk_norm_rope(q, k, pos, table, q_gain=gain, out=(q, k))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(v, kept)


def test_norm_rope_positions_outside_the_table_and_edges():
    q, k, _ = prompt_inputs([6], (4, 2, 64), F32, 71)
    q[2], k[2] = 0, 0                                            # a zero head stays zero
    q[3] = 1e-30
    pos = ints([0, -1, 5, 9, 10, 2 ** 31 - 1])
    one = torch.ones(64, device="cuda")
    qo, ko = ssq.ssq_qk_norm_rope(q, k, pos, rope_table(10, 64), q_gain=one, k_gain=one)
    assert torch.isnan(qo[[1, 4, 5]]).all() and torch.isnan(ko[[1, 4, 5]]).all()
    assert torch.isfinite(qo[[0, 2, 3]]).all() and not qo[2].any() and not ko[2].any()
    assert ssq.ssq_qk_norm_rope(q[:0], k[:0], pos[:0], rope_table(10, 64))[0].shape == (0, 4, 64)


# --- streams, graphs, refusals ------------------------------------------------------------------

def test_on_another_stream_and_in_a_graph():
    """A step of two layers' worth of calls, captured and replayed with new inputs in between."""
    heads, page, n, prefix = (16, 4, 64), 16, 5, 40
    lens = [60, 47, 90, 41, 55]
    q, k, v, table, _ = cache_inputs(lens, 1, prefix, page, heads, BF, 80, extra=2)
    free = ints([int(x) for x in range(k.shape[0])][::-1])
    dev, rope = table.cuda(), rope_table(256, 64)
    held, added = ints([x - 1 for x in lens]), ints([1] * n)
    new_k, new_v = (A.model_like(gen(81 + i), (n, 4, 64), BF) for i in range(2))
    ws = torch.empty(ssq.ssq_attention_decode_workspace_size(n, 1, 16, 4, 64, 128, prefix), dtype=torch.uint8, device="cuda")

    def step():
        _, ln, pos, slots, _, _ = ssq.ssq_page_tables(held, added, free, dev, page, n)
        qo, _ = ssq.ssq_qk_norm_rope(q[:, 0], new_k, pos, rope, v=new_v, slots=slots, k_pages=k, v_pages=v)
        return ssq.ssq_attention_decode(qo.view(n, 1, 16, 64), k, v, dev, ln, 128, prefix=prefix, workspace=ws)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        first = step()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(4):
        q.copy_(A.model_like(gen(90 + i), q.shape, BF))
        new_v.mul_(1.0 + i)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        assert torch.equal(got, step())
        assert not torch.equal(got, first)
        ref, size, eps = A.decode_reference(ssq.ssq_qk_norm_rope(q[:, 0], new_k, held, rope)[0].view(n, 1, 16, 64), k, v, table, lens, 128, prefix)
        A.check(got, ref, size, eps, f"replay {i}")


def test_prompt_in_a_graph():
    lens = [100, 30]
    q, k, v = prompt_inputs(lens, (8, 2, 128), BF, 85)
    starts = ints(A.starts_of(lens))
    ssq.ssq_attention_prompt(q, k, v, starts)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = ssq.ssq_attention_prompt(q, k, v, starts)
    for i in range(3):
        v.mul_(0.5 + i)
        starts[1] = 100 - 7 * i
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ssq.ssq_attention_prompt(q, k, v, starts))


def test_wrong_tensors_are_refused():
    q, k, v = prompt_inputs([20], (8, 2, 64), BF, 90)
    starts, pos, rope = ints([0, 20]), torch.arange(20, device="cuda", dtype=torch.int32), rope_table(32, 64)
    pools = [torch.zeros((4, 2, 16, 64), device="cuda", dtype=BF) for _ in "kv"]
    table, lens = ints([[0, 1]]), ints([20])
    with pytest.raises(TypeError):
        ssq.ssq_attention_prompt(q.half(), k.half(), v.half(), starts)
    for bad in ((q, k, v[:19], starts), (q, k.float(), v, starts), (q, k, v, starts.long()), (q, k[:, :, :32], v, starts),
                (q.transpose(0, 1), k, v, starts), (q, k, v, starts.cpu()), (q[..., ::2], k, v, starts)):
        with pytest.raises(ValueError):
            ssq.ssq_attention_prompt(*bad)
    with pytest.raises(ssq.SSQError):
        ssq.ssq_attention_prompt(q[:, :7], k, v, starts)                    # 7 heads on 2
    with pytest.raises(ssq.SSQError):
        ssq.ssq_attention_prompt(q, k, v, starts, scale=0.0)
    with pytest.raises(ValueError):
        ssq.ssq_qk_norm_rope(q, k, pos, rope, slots=pos)
    with pytest.raises(ValueError):
        ssq.ssq_qk_norm_rope(q, k, pos, rope[:, :32].contiguous())
    with pytest.raises(ValueError):
        ssq.ssq_qk_norm_rope(q, k, pos.long(), rope)
    d = q[:1].view(1, 1, 8, 64)
    for bad in ((d, pools[0], pools[1][:3], table, lens, 20), (d, pools[0].float(), pools[1].float(), table, lens, 20),
                (d, *pools, table[0], lens, 20), (d, *pools, table, lens.long(), 20), (d[0], *pools, table, lens, 20)):
        with pytest.raises(ValueError):
            ssq.ssq_attention_decode(*bad)
    with pytest.raises(ssq.SSQError):
        ssq.ssq_attention_decode(d, *pools, table, lens, -1)
    with pytest.raises(ssq.SSQError):
        ssq.ssq_page_tables(lens, lens, pos, table, 24, 5)
    with pytest.raises(ValueError):
        ssq.ssq_page_tables(lens, ints([1, 2]), pos, table, 16, 5)
