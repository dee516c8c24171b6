"""Joins of the parts of a decoded row, in every form: a wavefront or a workgroup a row, both head sizes, as many parts as
are held ahead and more.  Sampled rows in 64 bits, so that the shapes can be those of serving."""
import pytest
import torch

from paper_2607_08779_amd import ssq
from tests import attention_common as A
from tests.test_gpu_attention import BF, F32, gen, ints

pytestmark = pytest.mark.gpu

# requests, own lengths (fresh ones among them), fresh, prefix, heads, page; rows of out; parts at least, at most
JOINS = [
    (53, (1, 200), 1, 600, (30, 10, 128), 64, 1590, 2, 8),           # a wavefront a row, not a whole workgroup of them
    (23, (3, 90), 3, 515, (23, 1, 128), 16, 1587, 2, 16),
    (64, (1, 1024), 1, 8192, (32, 8, 128), 64, 2048, 17, 64),        # more parts than a wavefront holds ahead
    (51, (1, 300), 1, 8200, (31, 1, 128), 32, 1581, 17, 64),
    (3, (4000, 6000), 1, 16000, (8, 2, 128), 64, 24, 33, 64),        # a workgroup a row, more than it holds ahead
    (2, (3000, 3001), 2, 16005, (6, 6, 128), 16, 24, 33, 64),
    (1, (16383, 16383), 1, 0, (32, 8, 128), 64, 32, 17, 32),
    (24, (1, 100), 1, 200000, (64, 1, 64), 64, 1536, 33, 64),        # heads of 64
    (2, (5000, 5001), 1, 16384, (9, 3, 64), 32, 18, 33, 64),
    (40, (1, 100), 1, 2000, (39, 13, 64), 16, 1560, 2, 16),
]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("i", range(len(JOINS)))
def test_decode_joins(i, dtype):
    n, own, fresh, prefix, (hq, hk, d), page, rows, least, most = JOINS[i]
    g, pick = gen(600 + i), torch.Generator().manual_seed(600 + i)
    lens = [prefix + x for x in torch.randint(own[0], own[1] + 1, (n,), generator=pick).tolist()]
    lens[n // 2] = prefix + own[1]
    size = ssq.ssq_attention_decode_workspace_size(n, fresh, hq, hk, d, max(lens), prefix)
    parts, rest = divmod(size, rows * (8 + 4 * d))
    assert rows == n * fresh * hq and rest == 0 and least <= parts <= most, parts
    shared, need = prefix // page, [A.pages_for(x, page) for x in lens]
    pages = shared + sum(x - shared for x in need)
    ids, table, at = torch.randperm(pages, generator=pick), torch.full((n, max(need)), -1), shared
    for r in range(n):
        table[r, :shared] = ids[:shared]
        table[r, shared:need[r]] = ids[at:at + need[r] - shared]
        at += need[r] - shared
    k, v = (A.model_like(g, (pages * page, hk, d), dtype).view(pages, page, hk, d).transpose(1, 2).contiguous() for _ in "kv")
    q = A.model_like(g, (n, fresh, hq, d), dtype)
    out = ssq.ssq_attention_decode(q, k, v, table.int().cuda(), ints(lens), max(lens), prefix=prefix)
    for r in {0, 1 % n, n // 2, n - 1}:
        for head in {0, hk // 2, hk - 1}:
            kk, _ = A.gather(k, table[r], table[0], prefix, lens[r], head)
            vv, _ = A.gather(v, table[r], table[0], prefix, lens[r], head)
            for t in {0, fresh - 1}:
                for h in {head * (hq // hk), head * (hq // hk) + hq // hk - 1}:
                    ref = A.attend(q[r, t, h:h + 1], kk, vv, torch.tensor([lens[r] - fresh + t]), d ** -0.5)
                    A.check(out[r, t, h:h + 1], *ref, f"{JOINS[i]} {dtype} request {r} token {t} head {h}")
    assert torch.isfinite(out).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_prompt_rows_before_a_bad_token_of_the_same_tile(bad, dtype):
    """The rows of a sequence before its own bad token, which tokens of the sequences before it and later ones share."""
    from tests.test_gpu_attention import prompt_inputs
    lens = [70, 130, 45]
    q, k, v = prompt_inputs(lens, (8, 2, 128), dtype, 640, pad=9)
    ref, size, eps = A.prompt_reference(q, k, v, lens)
    for t in (41, 134, 171, 231, 246):                              # the first's, the second's two, the third's, padding
        k[t, :, ::3], v[t, :, 1::2] = bad, bad
    out = ssq.ssq_attention_prompt(q, k, v, ints(A.starts_of(lens)))
    for a, b in ((0, 41), (70, 134), (200, 231)):
        A.check(out[a:b], ref[a:b], size[a:b], eps[a:b], f"{bad} {a}")
        end = a + lens[(0, 70, 200).index(a)]
        assert not out[b:end].isfinite().all(-1).any()
    assert not out[245:].any()
