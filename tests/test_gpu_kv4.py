"""The 4-bit cache on the GPU: what a store writes, to the byte, and attention over it against 64 bits."""
import pytest
import torch

from oracle import ssq_oracle as O
from paper_2607_08779_amd import ssq
from tests import attention_common as A
from tests import kv4_common as Q
from tests.test_gpu_attention import BF, F32, cache_inputs, gen, ints

pytestmark = pytest.mark.gpu
NAN_SCALES = 0xFF              # as a byte of codes 15 and 15, as one of a binary16 scale NaN


def bits(x):
    return x.contiguous().view(torch.int16 if x.element_size() == 2 else torch.int32)


def new_cache(pages, heads, page, dim, fill=NAN_SCALES):
    cache = ssq.ssq_kv4_cache(pages, heads, page, dim)
    assert cache.shape == (pages, heads, 2, Q.part_bytes(page, dim)) and not cache.any()
    return cache.fill_(fill)


def check_store(k, v, slots, cache, before, page, held, tag):
    """Every byte of the cache, and the rows as held."""
    t, heads, dim = k.shape
    want = before.cpu().clone()
    for which, x in enumerate((k, v)):
        u, scale = Q.on_grid(x)
        byte, shift = Q.places(page, dim)[which]
        for i, slot in enumerate(slots.tolist()):
            if not 0 <= slot < cache.shape[0] * page:
                continue
            e, at = slot // page, slot % page
            for h in range(heads):
                part = want[e, h, which]
                part[byte[at]] = 0
                for d in range(dim):
                    part[byte[at, d]] |= int(u[i, h, d]) << int(shift[at, d])
                part[page * dim // 2:].view(torch.float16)[at * (dim // 32):(at + 1) * (dim // 32)] = scale[i, h]
        if held is not None:
            values = (u - 8).float() * scale.float().repeat_interleave(32, 2)
            assert torch.equal(torch.nan_to_num(held[which].cpu(), nan=77.0), torch.nan_to_num(values.to(x.dtype), nan=77.0)), f"{tag}: held {which}"
    got = cache.cpu()
    nan = (got != want).nonzero()
    assert len(nan) == 0, f"{tag}: {len(nan)} bytes differ, first at {nan[0].tolist()}"


STORES = [
    # tokens, kv_heads, dim, page
    (1, 8, 128, 64), (1, 1, 64, 16), (3, 2, 64, 16), (17, 8, 128, 32), (70, 3, 64, 128), (33, 5, 128, 1024), (131, 1, 128, 16),
]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("i", range(len(STORES)))
def test_store(i, dtype):
    t, heads, dim, page = STORES[i]
    g = gen(600 + i)
    q, k, v = A.model_like(g, (t, heads + 2, dim), dtype), A.model_like(g, (t, heads, dim), dtype), A.model_like(g, (t, heads, dim), dtype)
    if i % 2:                                    # rows of one projection
        k, v = torch.cat((q, k, v), 1).split((heads + 2, heads, heads), 1)[1:]
    pages = A.pages_for(t, page) + 2
    slots = torch.randperm(pages * page, generator=g, device="cuda")[:t].to(torch.int32)
    if t > 2:
        slots[1], slots[t - 1] = -1, pages * page
    cache = new_cache(pages, heads, page, dim)
    before = cache.clone()
    held = ssq.ssq_kv4_store(k, v, slots, cache, held=i % 3 != 0)
    assert (held is None) == (i % 3 == 0)
    check_store(k, v, slots, cache, before, page, held, f"{STORES[i]} {dtype}")


@pytest.mark.parametrize("dtype", [BF, F32])
def test_store_grid_is_that_of_the_weights(dtype):
    """Codes and scales of ssq_quantize (signed grid, 4 bits, groups of 32), which the oracle pins."""
    t, heads, dim, page = 40, 4, 128, 64
    k = A.model_like(gen(620), (t, heads, dim), dtype)
    cache = new_cache(1, heads, page, dim)
    ssq.ssq_kv4_store(k, k, torch.arange(t, device="cuda", dtype=torch.int32), cache)
    ref = O.quantize(k.float().cpu().numpy().reshape(t * heads, dim), 32, 4, O.SIGNED_SYM)
    codes = torch.from_numpy(ref.codes).view(t, heads, dim // 2)
    want = torch.stack((codes & 15, codes >> 4), -1).flatten(2).to(torch.int32)
    for u, s in Q.read(cache, page, dim):
        assert torch.equal(u[0, :, :t].transpose(0, 1), want)
        assert torch.equal(bits(s[0, :, :t].transpose(0, 1).half()), torch.from_numpy(ref.scales.view("int16")).view(t, heads, dim // 32))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_store_of_odd_groups(dtype):
    """Zeros, ties between signs, halves between steps, the smallest and largest numbers, infinities and NaN."""
    dim, page = 64, 16
    rows = torch.zeros((12, 1, dim))
    rows[1, 0, :32] = 3.0
    rows[2, 0, 5], rows[2, 0, 9] = 4.0, -4.0                              # a tie: the scale is positive
    rows[3, 0, :32] = torch.arange(32) / 2.0 - 8.0                        # halves: to even
    rows[4, 0, :32] = 8.0 - torch.arange(32) / 2.0
    rows[5, 0, 0], rows[5, 0, 40] = float("nan"), 1.0
    rows[6, 0, 31], rows[6, 0, 32] = float("inf"), -float("inf")
    rows[7, 0, :4] = torch.tensor([524160.0, 1.0, -2.0, 3.0])             # s = 65520 rounds to infinity
    rows[8, 0, :4] = torch.tensor([-522240.0, 1.0, -2.0, 300000.0])       # the largest that binary16 reaches in bf16
    rows[9, 0, :3] = torch.tensor([1e-7, -3e-8, 2e-9])                    # scales below the normal numbers
    rows[10, 0, :3] = torch.tensor([1e-40, -3e-39, 0.0])
    rows[11, 0, ::2] = -0.0
    k = rows.to(dtype).cuda()
    cache = new_cache(1, 1, page, dim, 0)
    before = cache.clone()
    slots = torch.arange(12, device="cuda", dtype=torch.int32)
    held = ssq.ssq_kv4_store(k, -k, slots, cache, held=True)
    check_store(k, -k, slots, cache, before, page, held, str(dtype))
    assert held[0][5, 0, :32].isnan().all() and held[0][5, 0, 32:].isfinite().all() and held[0][7, 0, :32].isnan().all()
    assert held[0][8].isfinite().all()


def test_store_of_groups_near_the_smallest_numbers():
    """Binary32 groups whose scale is below the normal numbers, rounded or zero: quotients beyond both ends of the grid
    are clipped, every code is that of ssq_quantize_f32, and what is held is zero, as binary16 has no such scale."""
    dim, page, heads, tokens = 64, 64, 2, 128
    g = torch.Generator().manual_seed(640)
    tiny = 2.0 ** -149
    size = torch.tensor([*range(1, 101), *(1 << n for n in range(7, 32)), 3, 11, 12], dtype=torch.float64)
    k = torch.rand((tokens, heads, dim), generator=g, dtype=torch.float64) * 2 - 1
    k[:, 1] = k[:, 1].sign() * (torch.rand((tokens, dim), generator=g) < 0.3)      # ends of the grid, and zeros
    k[:, :, 7], k[:, :, 40] = 1.0, -1.0                                    # the largest of their groups
    k = ((k * size[:, None, None]).round() * tiny).float()
    assert (k[:, :, 7].double() == size[:, None] * tiny).all()
    rows = k.cuda(), (-k).cuda()
    cache = new_cache(2, heads, page, dim)
    held = ssq.ssq_kv4_store(*rows, torch.arange(tokens, device="cuda", dtype=torch.int32), cache, held=True)
    for x, h, (u, s) in zip(rows, held, Q.read(cache, page, dim)):
        assert (h == 0).all() and (s == 0).all()
        codes, scales, _ = ssq.ssq_quantize(x.reshape(tokens * heads, dim), 32, 4, ssq.SIGNED_SYM)
        codes = codes.cpu().view(tokens, heads, dim // 2)
        got = u.permute(0, 2, 1, 3).reshape(tokens, heads, dim)
        assert torch.equal(got, torch.stack((codes & 15, codes >> 4), -1).flatten(2).to(torch.int32))
        assert torch.equal(bits(s.permute(0, 2, 1, 3).reshape(tokens * heads, 2).half()), scales.cpu())
        # and the definition, wherever the quotient is a number: s as binary32 rounds it
        w = x.cpu().double().unflatten(2, (-1, 32))
        hi, down = w.amax(3, keepdim=True), -w.amin(3, keepdim=True)
        step = (torch.maximum(hi, down) / 8).float().double()
        c = (w / torch.where(hi > down, -step, step)).float().round().clamp(-8, 7)
        known = ~c.isnan()
        assert torch.equal(got.unflatten(2, (-1, 32))[known], (c[known] + 8).to(torch.int32))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_store_in_place_and_into_strided_rows(dtype):
    t, heads, dim, page = 29, 3, 64, 16
    k, v = (A.model_like(gen(630 + i), (t, heads, dim), dtype) for i in range(2))
    slots = torch.arange(t, device="cuda", dtype=torch.int32)
    cache, other = (new_cache(2, heads, page, dim) for _ in range(2))
    want = ssq.ssq_kv4_store(k, v, slots, cache, held=True)
    wide = torch.full((t, 2 * heads + 2, dim), 7.0, dtype=dtype, device="cuda")
    ssq.ssq_kv4_store(k, v, slots, other, held=(wide[:, 1:1 + heads], wide[:, 1 + heads:1 + 2 * heads]))
    assert torch.equal(wide[:, 1:1 + heads], want[0]) and torch.equal(wide[:, 1 + heads:-1], want[1]) and (wide[:, ::2 * heads + 1] == 7).all()
    ssq.ssq_kv4_store(k, v, slots, other, held=(k, v))
    assert torch.equal(k, want[0]) and torch.equal(v, want[1]) and torch.equal(cache, other)
    again = ssq.ssq_kv4_store(k, v, slots, other, held=True)             # held rows are on the grid: nothing changes
    if dtype == F32:
        assert torch.equal(again[0], k)
    assert ssq.ssq_kv4_store(k[:0], v[:0], slots[:0], cache) is None and torch.equal(ssq.ssq_kv4_store(k[:0], v[:0], slots[:0], cache, held=True)[0], k[:0])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_store_rows_between_each_other(dtype):
    """Rows of all four arrays in one buffer, in equal and in different strides; keys that are the values, in place."""
    t, heads, dim, page = 9, 2, 64, 16
    k, v = (A.model_like(gen(635 + i), (t, heads, dim), dtype) for i in range(2))
    slots = torch.arange(t, device="cuda", dtype=torch.int32)
    cache = new_cache(1, heads, page, dim)
    want = ssq.ssq_kv4_store(k, v, slots, cache, held=True)
    cells = torch.full((12 * t, heads, dim), 7.0, dtype=dtype, device="cuda")
    # first cell and step of k, v, k_held, v_held; the last ones in place
    for places in (((0, 4), (1, 4), (2, 4), (3, 4)), ((3, 4), (2, 4), (1, 4), (0, 4)), ((0, 8), (2, 8), (1, 4), (3, 4)), ((1, 2), (60, 1), (0, 6), (25, 2)),
                   ((5, 4), (4, 6), (5, 4), (4, 6))):
        cells.fill_(7.0)
        rows = [cells[a:a + t * s:s] for a, s in places]
        rows[0].copy_(k), rows[1].copy_(v)
        seen = [set(range(a, a + t * s, s)) for a, s in places]
        if places[0] != places[2]:
            assert sum(map(len, seen)) == len(set.union(*seen)), "the places are apart"
        other = new_cache(1, heads, page, dim)
        ssq.ssq_kv4_store(rows[0], rows[1], slots, other, held=(rows[2], rows[3]))
        assert torch.equal(rows[2], want[0]) and torch.equal(rows[3], want[1]) and torch.equal(other, cache), places
        rest = [i for i in range(len(cells)) if i not in set.union(*seen)]
        assert (cells[rest] == 7).all()
    both = ssq.ssq_kv4_store(k, k, slots, cache, held=True)
    same = k.clone()
    ssq.ssq_kv4_store(same, same, slots, other, held=(same, same))
    assert torch.equal(both[0], both[1]) and torch.equal(same, both[0]) and torch.equal(cache, other)


# --- decoding -----------------------------------------------------------------------------------

def kv4_inputs(lens, fresh, prefix, page, heads, dtype, seed, extra=0):
    """As cache_inputs, in 4 bits; slots that no request should see have NaN scales, codes 15."""
    q, k, v, table, lens = cache_inputs(lens, fresh, prefix, page, heads, dtype, seed, poison=float("nan"), extra=extra)
    pages = k.shape[0]
    rows = [x.transpose(1, 2).reshape(pages * page, heads[1], heads[2]) for x in (k, v)]
    slots = torch.arange(pages * page, device="cuda", dtype=torch.int32)
    slots[rows[0][:, 0, 0].isnan()] = -1
    cache = new_cache(pages, heads[1], page, heads[2])
    ssq.ssq_kv4_store(*rows, slots, cache)
    return q, cache, table, lens


def run(q, cache, table, lens, prefix, max_len=None, **more):
    return ssq.ssq_attention_decode_kv4(q, cache, table.cuda(), ints(lens), max(lens) if max_len is None else max_len, prefix=prefix, **more)


DECODES = [
    # lens, fresh, prefix, page, heads
    ([1], 1, 0, 16, (4, 4, 64)),
    ([33, 1, 64, 500], 1, 0, 16, (32, 8, 128)),
    ([0, 5, 0], 1, 0, 16, (8, 2, 64)),
    ([1700], 1, 0, 64, (40, 8, 128)),
    ([100, 130, 101], 1, 100, 16, (32, 8, 128)),           # a prefix that ends inside a page
    ([96, 100, 97, 160, 96], 1, 96, 32, (14, 2, 64)),
    ([300, 40, 333, 0], 1, 297, 64, (8, 1, 128)),          # shorter than the prefix
    ([270 + i for i in range(20)], 1, 257, 16, (8, 2, 128)),
    ([70 + 9 * i for i in range(40)], 2, 64, 16, (16, 4, 64)),
    ([10, 3, 1, 0, 25], 4, 0, 16, (8, 2, 128)),            # tokens before the first key
    ([150, 170], 9, 120, 32, (32, 4, 64)),                 # more rows than a tile
    ([600, 650, 700], 3, 512, 128, (6, 6, 128)),
    ([50, 60], 1, 40, 1024, (130, 1, 64)),
    ([1100, 1030], 1, 1024, 16, (8, 8, 64)),
    ([31, 32, 33, 15, 16, 17, 47, 48, 49], 1, 15, 16, (4, 2, 64)),
    ([127, 128, 129, 255, 256, 257], 1, 0, 32, (3, 3, 128)),
    ([520, 470], 6, 300, 16, (20, 4, 128)),                # 30 rows a key/value head
    ([90, 100, 95], 3, 64, 16, (16, 4, 128)),              # 12 rows
    ([2900], 1, 0, 64, (16, 1, 128)),                      # 16 rows, in parts
    ([2500, 1700], 4, 0, 32, (10, 2, 128)),                # 20 rows, in parts
    ([1900, 2300], 3, 0, 16, (12, 6, 64)),                 # 6 rows, in parts
    ([350 + 11 * i for i in range(33)], 1, 333, 32, (7, 1, 128)),
]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("i", range(len(DECODES)))
def test_decode(i, dtype):
    lens, fresh, prefix, page, heads = DECODES[i]
    q, cache, table, lens = kv4_inputs(lens, fresh, prefix, page, heads, dtype, 640 + i)
    ref, bound = Q.decode_reference(q, cache, page, table, lens, max(lens), prefix)
    for name, more in (("workspace", {}), ("none", {"workspace": torch.empty(0, dtype=torch.uint8, device="cuda")})):
        print(DECODES[i], dtype, name, flush=True)
        Q.check(run(q, cache, table, lens, prefix, **more), ref, bound, f"{DECODES[i]} {dtype} {name}")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("prefix", [0, 90])
def test_decode_absent_pages(dtype, prefix):
    lens = [200, 230, 190]
    q, cache, table, lens = kv4_inputs(lens, 1, prefix, 16, (8, 2, 64), dtype, 660)
    table[1, 9], table[2, 6], table[2, 11] = -1, cache.shape[0], 2 ** 31 - 1
    if prefix:
        table[:, 2] = -5
    ref, bound = Q.decode_reference(q, cache, 16, table, lens, 230, prefix)
    for ws in (None, torch.empty(0, dtype=torch.uint8, device="cuda")):
        Q.check(run(q, cache, table, lens, prefix, workspace=ws), ref, bound, f"absent {prefix}")


def test_decode_all_pages_absent_or_no_pages():
    q, cache, table, lens = kv4_inputs([40, 50], 1, 0, 16, (8, 2, 64), BF, 661)
    assert not run(q, cache, torch.full_like(table, -1), lens, 0).any()
    assert not run(q, cache[:0], table, lens, 0).any()
    assert not run(q, cache, table[:, :0].contiguous(), lens, 0).any()
    assert not run(q, cache, table, [0, -3], 0, max_len=50).any()
    assert not run(q, cache, table, lens, 0, max_len=0).any()
    assert run(q[:0], cache, table[:0], [], 0, max_len=5).shape == (0, 1, 8, 64)


def test_decode_lengths_are_bounded():
    q, cache, table, _ = kv4_inputs([500, 90], 1, 0, 16, (8, 2, 64), BF, 662)
    for max_len, width in ((120, table.shape[1]), (500, 3), (2 ** 30, 4), (100000, table.shape[1])):
        t = table[:, :width].contiguous()
        ref, bound = Q.decode_reference(q, cache, 16, t, [500, 90], max_len, 0)
        Q.check(run(q, cache, t, [500, 90], 0, max_len=max_len), ref, bound, f"{max_len} {width}")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("prefix", [0, 70])
def test_decode_requests_of_all_lengths(prefix, dtype):
    """More requests than places: empty, equal and long ones."""
    some = [0, 700, 33, 700, 1, 64, 699, 5, 128, 0, 300]
    lens = [0 if some[r % 11] == 0 else prefix + some[r % 11] - r % 3 * (some[r % 11] > 9) for r in range(131)]
    q, cache, table, _ = kv4_inputs(lens, 1, prefix, 64, (6, 3, 64), dtype, 663)
    ref, bound = Q.decode_reference(q, cache, 64, table, lens, max(lens), prefix)
    Q.check(run(q, cache, table, lens, prefix), ref, bound, f"{prefix} {dtype}")


@pytest.mark.parametrize("factor", [0.0, 30.0, 1e4])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_decode_flat_and_sharp_scores(factor, dtype):
    lens = [140, 700]
    q, cache, table, lens = kv4_inputs(lens, 1, 0, 16, (8, 2, 128), dtype, 664)
    q = (q.float() * factor).to(dtype)
    Q.check(run(q, cache, table, lens, 0), *Q.decode_reference(q, cache, 16, table, lens, max(lens), 0), f"factor {factor}")
    q, cache, table, lens = kv4_inputs(lens, 1, 100, 16, (8, 2, 128), dtype, 665)
    q = (q.float() * factor).to(dtype)
    Q.check(run(q, cache, table, lens, 100), *Q.decode_reference(q, cache, 16, table, lens, max(lens), 100), f"factor {factor}")


@pytest.mark.parametrize("factor", [4.0, 4096.0])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("prefix", [0, 100])
def test_decode_sharp_scores_give_the_winners_value(prefix, dtype, factor):
    """Keys and values that the grid holds exactly, queries along one key that each sees: all other weights are below
    e^-200, so that a row is that key's value, whatever the scores' size.  Off by: in bf16 weight times scale rounded and
    the row rounded (2^-8 each), and codes' offsets in at most 64 terms below 279 scales; in binary32 ten roundings."""
    fresh, page, (hq, hk, d) = 3, 16, (8, 2, 128)
    q, cache, table, lens = kv4_inputs([700, 140, 1500], fresh, prefix, page, (hq, hk, d), dtype, 673)
    g = torch.Generator().manual_seed(674)
    shape = (cache.shape[0] * page, hk, d // 32, 32)
    k, v = (torch.randint(-8, 8, shape, generator=g).float() for _ in "kv")
    for x in (k, v):
        x.scatter_(3, torch.randint(0, 32, (*shape[:3], 1), generator=g), -8.0)      # the step is 1
        x *= 1 - 2.0 * torch.randint(0, 2, (*shape[:3], 1), generator=g)             # or -1
    size = torch.ldexp(torch.ones(()), torch.randint(-6, 7, (*shape[:3], 1), generator=g))
    k, v, step = k.flatten(2), (v * size).flatten(2), size.expand(shape).flatten(2)
    held = ssq.ssq_kv4_store(k.to(dtype).cuda(), v.to(dtype).cuda(), torch.arange(shape[0], device="cuda", dtype=torch.int32), cache, held=True)
    assert torch.equal(held[0].cpu().float(), k) and torch.equal(held[1].cpu().float(), v)
    want, tol = (torch.zeros(q.shape, dtype=torch.float64) for _ in range(2))
    for r, n in enumerate(lens):
        at = torch.arange(n)
        slot = torch.where(at < prefix, table[0, at // page], table[r, at // page]) * page + at % page
        for i in range(fresh):
            seen = n - fresh + i + 1
            for h in range(hq):
                kv = h * hk // hq
                w = (0, seen - 1, max(prefix - 1, 0), int(torch.randint(0, seen, (), generator=g)))[(h + i) % 4]
                row = factor * k[slot[w], kv]
                score = (k[slot[:seen], kv].double() * row.double()).sum(1) * d ** -0.5
                rest = torch.cat((score[:w], score[w + 1:]))
                assert score[w] - rest.max() > 200
                q[r, i, h] = row.to(dtype)
                want[r, i, h] = v[slot[w], kv].double()
                tol[r, i, h] = 2.0 ** -7 * want[r, i, h].abs() + 64 * 279 * Q.U * step[slot[w], kv] if dtype == BF else 10 * Q.U * want[r, i, h].abs()
    for ws in (None, torch.empty(0, dtype=torch.uint8, device="cuda")):
        Q.check(run(q, cache, table, lens, prefix, workspace=ws), want, tol, f"{prefix} {dtype} {factor}")


CHUNKS = [
    # as DECODES: many new tokens at once, whose last tile of rows is partly empty
    ([400], 150, 0, 16, (8, 2, 64)), ([131], 131, 0, 32, (3, 3, 64)), ([333, 290], 40, 200, 64, (10, 2, 128)), ([20, 200, 90], 130, 0, 16, (4, 4, 64)),
]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("i", range(len(CHUNKS)))
def test_decode_of_many_new_tokens(i, dtype):
    lens, fresh, prefix, page, heads = CHUNKS[i]
    q, cache, table, lens = kv4_inputs(lens, fresh, prefix, page, heads, dtype, 676 + i)
    ref, bound = Q.decode_reference(q, cache, page, table, lens, max(lens), prefix)
    for ws in (None, torch.empty(0, dtype=torch.uint8, device="cuda")):
        Q.check(run(q, cache, table, lens, prefix, workspace=ws), ref, bound, f"{CHUNKS[i]} {dtype}")


@pytest.mark.parametrize("sign", [1, -1])
def test_decode_rising_and_falling_scores(sign):
    """Each key outscores all before it by far: the running reference moves at every tile."""
    n, d, page = 900, 64, 16
    v = A.model_like(gen(666), (n, 1, d), BF)
    k = (sign * torch.arange(n, device="cuda", dtype=F32) * 0.25)[:, None, None].expand(n, 1, d).to(BF).contiguous()
    cache = new_cache(A.pages_for(n, page), 1, page, d)
    ssq.ssq_kv4_store(k, v, torch.arange(n, device="cuda", dtype=torch.int32), cache)
    table, q = torch.arange(cache.shape[0], dtype=torch.int32)[None], torch.ones((1, 1, 2, d), device="cuda", dtype=BF)
    Q.check(run(q, cache, table, [n], 0), *Q.decode_reference(q, cache, page, table, [n], n, 0), f"{sign}")


@pytest.mark.parametrize("dtype", [BF, F32])
def test_decode_one_sided_values_in_flat_attention(dtype):
    """All values of one sign, whose codes' offsets would add up over the keys if they were not taken out with them;
    and values whose mean is far below their size."""
    n, d, page = 2000, 128, 32
    g = gen(667)
    k = A.model_like(g, (n, 2, d), dtype)
    for v in (A.model_like(g, (n, 2, d), dtype).abs(), A.model_like(g, (n, 2, d), dtype)):
        v[:, 0, ::32] = v[:, 0].amax() * 2           # every scale of the first head negative
        cache = new_cache(A.pages_for(n, page), 2, page, d)
        ssq.ssq_kv4_store(k, v, torch.arange(n, device="cuda", dtype=torch.int32), cache)
        table, q = torch.arange(cache.shape[0], dtype=torch.int32)[None], A.model_like(g, (1, 1, 4, d), dtype) * 0.01
        Q.check(run(q, cache, table, [n], 0), *Q.decode_reference(q, cache, page, table, [n], n, 0), f"{dtype}")


def test_decode_strided_queries_and_given_buffers():
    lens, heads = [150, 90, 200], (8, 2, 128)
    q, cache, table, lens = kv4_inputs(lens, 2, 64, 16, heads, BF, 668)
    ref, bound = Q.decode_reference(q, cache, 16, table, lens, 200, 64)
    wide = torch.cat((q, torch.full_like(q, float("nan"))), 2)           # rows of a fused projection
    size = ssq.ssq_attention_decode_kv4_workspace_size(3, 2, 8, 2, 128, 200, 64)
    assert size > 0
    ws, out = torch.full((size + 256,), 0xFF, dtype=torch.uint8, device="cuda"), torch.empty_like(q)
    first = run(wide[:, :, :8], cache, table, lens, 64, workspace=ws, out=out)
    assert first is out and (ws[size:] == 0xFF).all()
    Q.check(out, ref, bound, "strided")
    again = run(q, cache, table, lens, 64)
    assert torch.equal(bits(out), bits(again))
    ref, bound = Q.decode_reference(q, cache, 16, table, lens, 200, 64, scale=0.3)
    Q.check(run(q, cache, table, lens, 64, scale=0.3), ref, bound, "scale")


@pytest.mark.parametrize("dtype", [BF, F32])
def test_decode_values_that_are_nan_reach_the_rows_that_see_them(dtype):
    """A NaN in a key makes the rows that see it NaN; one in a value the 32 elements of its group."""
    n, page, heads = 100, 16, (4, 2, 64)
    g = gen(669)
    k, v = (A.model_like(g, (n, 2, 64), dtype) for _ in "kv")
    k[95, 1, 3], v[97, 0, 40] = float("nan"), float("inf")
    cache = new_cache(7, 2, page, 64)
    ssq.ssq_kv4_store(k, v, torch.arange(n, device="cuda", dtype=torch.int32), cache)
    table, q = torch.arange(7, dtype=torch.int32)[None], A.model_like(g, (1, 8, 4, 64), dtype)
    out = run(q, cache, table, [n], 0)[0]                                # positions 92..99
    assert out[:3].isfinite().all() and out[3:, 2:].isnan().all() and out[:5, :2].isfinite().all()
    assert out[5:, :2, 32:].isnan().all() and out[5:, :2, :32].isfinite().all()


def test_decode_of_as_many_requests_as_a_launch_holds():
    """2^20 requests of 15 heads, a workgroup each: those of no token give zeros, of one token its value."""
    n, heads, d, page = 1 << 20, 15, 64, 16
    g = gen(675)
    k, v = (torch.randn((4 * page, heads, d), generator=g, device="cuda").bfloat16() for _ in "kv")
    cache = new_cache(4, heads, page, d)
    _, held = ssq.ssq_kv4_store(k, v, torch.arange(4 * page, device="cuda", dtype=torch.int32), cache, held=True)
    q = torch.randn((n, 1, heads, d), generator=g, device="cuda", dtype=BF)
    request = torch.arange(n, device="cuda", dtype=torch.int32)
    lens, table = request % 2, (request % 4)[:, None].contiguous()
    out = ssq.ssq_attention_decode_kv4(q, cache, table, lens, page)
    assert not out[::2].any()
    for r in (1, 3):                               # weight times scale, and the quotient, rounded once each
        want = held[page * r].float()
        assert ((out[r::4, 0].float() - want).abs() <= 2.0 ** -7 * want.abs()).all()


# --- a row is a function of what it sees ----------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("prefix", [0, 64, 70])
def test_decode_row_does_not_depend_on_what_it_does_not_see(prefix, dtype):
    """To the bit: other requests' queries, later drafts, and every byte of the cache behind a draft's position."""
    fresh, page, heads = 5, 16, (16, 2, 128)
    q, cache, table, lens = kv4_inputs([130, 97, 200], fresh, prefix, page, heads, dtype, 670)
    q = (q.float() * 4).to(dtype)
    out = run(q, cache, table, lens, prefix)
    for fill in (0, 0x7C, 0xFC, 0xFF):             # codes and scales of zeros, infinities, NaN
        q2, c2 = (q.float() * -3).to(dtype), cache.clone()
        q2[:, :3] = q[:, :3]
        view = [c2[:, :, 0, :page * 64].unflatten(2, (page, 64)), c2[:, :, 1, :page * 64].unflatten(2, (page // 4, 64, 4)),
                *(c2[:, :, w, page * 64:].unflatten(2, (page, 8)) for w in (0, 1))]
        for r, n in enumerate(lens):
            for t in (n - 2, n - 1):                        # the last two of five
                e, at = int(table[r, t // page]), t % page
                view[0][e, :, at] = view[2][e, :, at] = view[3][e, :, at] = fill
                view[1][e, :, at // 4, :, at % 4] = fill
        again = run(q2, c2, table, lens, prefix)
        assert torch.equal(bits(again[:, :3]), bits(out[:, :3])), f"fill {fill}"
    q2 = (q.float() * 7).to(dtype)
    q2[1] = q[1]
    assert torch.equal(bits(run(q2, cache, table, lens, prefix)[1]), bits(out[1]))


def test_decode_long_cache_at_far_pages():
    """A cache of more than 2^32 bytes: pages at its far end, and a request of many tokens there."""
    page, heads, d = 1024, 8, 128
    pages = (1 << 32) // (heads * 2 * Q.part_bytes(page, d)) + 40
    cache = new_cache(pages, heads, page, d)
    g = gen(680)
    n = 3500
    k, v = (A.model_like(g, (n, heads, d), BF) for _ in "kv")
    ids = torch.tensor([pages - 1, 0, pages - 9, pages - 2], dtype=torch.int32)
    t = torch.arange(n, device="cuda")
    slots = (ids.cuda()[t // page] * page + t % page).to(torch.int32)
    ssq.ssq_kv4_store(k, v, slots, cache)
    q = A.model_like(g, (1, 1, 8, d), BF)
    out = run(q, cache, ids[None], [n], 0)
    few = cache[ids.long().cuda()]
    ref, bound = Q.decode_reference(q, few, page, torch.arange(4, dtype=torch.int32)[None], [n], n, 0)
    Q.check(out, ref, bound, "far pages")


# --- streams and graphs ----------------------------------------------------------------------------

def test_store_and_decode_in_a_replayed_graph():
    """A step captured once and replayed with new tokens, other work between the replays; a workspace of its own."""
    page, heads, d, n = 16, (8, 2, 64), 64, 3
    lens = [60, 34, 200]                                           # the new token has room in its request's last page
    q, cache, table, _ = kv4_inputs([x - 1 for x in lens], 1, 0, page, heads, BF, 690)
    table = table.cuda()
    k, v = (torch.empty((n, 2, d), dtype=BF, device="cuda") for _ in "kv")
    slots = torch.tensor([int(table[r, (x - 1) // page]) * page + (x - 1) % page for r, x in enumerate(lens)], dtype=torch.int32, device="cuda")
    dev_lens, out = ints(lens), torch.empty_like(q)
    ws = torch.empty(max(1, ssq.ssq_attention_decode_kv4_workspace_size(n, 1, 8, 2, d, 200)), dtype=torch.uint8, device="cuda")
    step = lambda to: (ssq.ssq_kv4_store(k, v, slots, cache, held=(k, v)),
                       ssq.ssq_attention_decode_kv4(q, cache, table, dev_lens, 200, out=to, workspace=ws))
    k.zero_(), v.zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(out)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out)
    for i in range(4):
        new = [A.model_like(gen(691 + i + 10 * j), (n, 2, d), BF) for j in range(2)]
        fresh = A.model_like(gen(695 + i), q.shape, BF)
        q.copy_(fresh)
        k.copy_(new[0]), v.copy_(new[1])
        graph.replay()
        got, held = out.clone(), (k.clone(), v.clone())
        torch.cuda.synchronize()
        k.copy_(new[0]), v.copy_(new[1])
        want = torch.empty_like(out)
        step(want)
        assert torch.equal(got, want) and torch.equal(held[0], k) and torch.equal(held[1], v), f"replay {i}"
        Q.check(got, *Q.decode_reference(q, cache, page, table.cpu(), lens, 200, 0), f"replay {i}")


def test_two_streams_at_once():
    a = [kv4_inputs([900, 300], 1, 0, 16, (8, 2, 128), BF, 700 + i) for i in range(2)]
    want = [run(q, c, t, n, 0) for q, c, t, n in a]
    tables, lens = [t.cuda() for _, _, t, _ in a], [ints(n) for *_, n in a]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in a], [None, None]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i] = ssq.ssq_attention_decode_kv4(a[i][0], a[i][1], tables[i], lens[i], 900)
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
