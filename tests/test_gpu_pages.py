"""Forks, free pages, compaction and copies of pages against lists, and all of them together as they are used."""
import random

import pytest
import torch

from paper_2607_08779_amd import ssq
from tests import attention_common as A
from tests import kv4_common as Q
from tests.test_gpu_attention import BF, F32, gen, ints

pytestmark = pytest.mark.gpu


def fork_reference(parents, lens, table, free, taken, page, width):
    out, lens_out, src, dst, seen = [], [], [], [], set()
    for p in parents:
        there = 0 <= p < len(lens)
        n_tokens = max(lens[p], 0) if there else 0
        n = -(-n_tokens // page)
        row = [table[p][j] if there and j < n and j < len(table[p]) else -1 for j in range(width)]
        s = d = -1
        if there and p in seen and n_tokens % page and n <= min(width, len(table[p])) and table[p][n - 1] >= 0:
            d = free[taken] if 0 <= taken < len(free) else -1
            s = table[p][n - 1] if d >= 0 else -1
            row[n - 1] = d
            taken += 1
        seen.add(p)
        out.append(row), lens_out.append(n_tokens), src.append(s), dst.append(d)
    return out, lens_out, src, dst, [taken]


def held_reference(lens, table, page, pages, pinned):
    held = {i for i in range(pages) if pinned and pinned[i]}
    for n, row in zip(lens, table):
        held |= {e for e in row[:-(-max(n, 0) // page)] if 0 <= e < pages}
    return held


def collect_reference(lens, table, page, pages, pinned=None):
    held = held_reference(lens, table, page, pages, pinned)
    free = [i for i in range(pages) if i not in held]
    return free + [-1] * (pages - len(free)), [len(free)]


def compact_reference(lens, table, page, pages, pinned=None):
    held = held_reference(lens, table, page, pages, pinned)
    used = len(held)
    holes = [i for i in range(used) if i not in held]
    movers = [i for i in range(used, pages) if i in held and not (pinned and pinned[i])]
    to = dict(zip(movers, holes))
    out = [[to.get(e, e) if j < -(-max(n, 0) // page) else e for j, e in enumerate(row)] for n, row in zip(lens, table)]
    after = (held - set(to)) | set(to.values())
    free = [i for i in range(pages) if i not in after]
    pad = [-1] * (pages // 2 - len(to))
    return out, free + [-1] * (pages - len(free)), [len(free)], movers + pad, [to[m] for m in movers] + pad, [len(to)]


def same(got, want, tag):
    for i, (g, w) in enumerate(zip(got, want)):
        assert g.dtype == torch.int32 and g.tolist() == w, f"{tag}: output {i}"


def random_table(rng, lens, width, pool, absent=0.0):
    return [[rng.choice((-1, -9)) if rng.random() < absent else rng.randrange(pool) for _ in range(width)] for _ in lens]


FORKS = [
    # rows, requests, longest, page, width, width out, free pages, taken
    (1, 1, 40, 16, 4, None, 3, 0), (1, 7, 40, 16, 4, None, 9, 2), (5, 0, 40, 16, 4, None, 3, 1), (0, 4, 1, 16, 3, None, 3, 0),
    (4, 16, 100, 16, 7, 9, 40, 0), (8, 17, 100, 32, 4, 3, 40, 5), (40, 33, 0, 16, 2, None, 4, 0), (64, 64, 500, 64, 9, None, 64, 3),
    (100, 1000, 3000, 16, 200, None, 700, 0), (300, 333, 70, 64, 1, None, 20, 0), (16384, 16384, 33, 16, 3, None, 9000, 11), (3, 50, 90, 16, 0, None, 5, 0),
    (9, 1040, 20, 16, 2, 5, 5000, 2000),
]


@pytest.mark.parametrize("i", range(len(FORKS)))
def test_fork(i):
    rows, requests, longest, page, width, width_out, count, taken = FORKS[i]
    rng = random.Random(800 + i)
    lens = [rng.choice((rng.randint(-1, longest), page * rng.randint(0, longest // page))) for _ in range(rows)]
    table = random_table(rng, lens, width, 10000, 0.05)
    parents = [rng.randint(-2, rows + 1) if rng.random() < 0.2 else rng.randrange(max(rows // 3, 1)) for _ in range(requests)]
    free = rng.sample(range(20000), count)
    got = ssq.ssq_page_fork(ints(parents), ints(lens), ints(table).view(rows, width), ints(free), page, taken=ints([taken]), width=width_out)
    want = fork_reference(parents, lens, table, free, taken, page, width if width_out is None else width_out)
    if requests and want[0][0]:
        same(got, want, FORKS[i])
    else:
        same(got[1:], want[1:], FORKS[i])
    out = [torch.full_like(x, 55) for x in got]
    again = ssq.ssq_page_fork(ints(parents), ints(lens), ints(table).view(rows, width), ints(free), page, taken=ints([taken]), out=out)
    assert all(x is y and torch.equal(x, z) for x, y, z in zip(again, out, got))


def test_fork_from_the_first_free_page():
    got = ssq.ssq_page_fork(ints([0, 0, 0]), ints([5]), ints([[3]]), ints([7, 8, 9]), 16)
    same(got, fork_reference([0, 0, 0], [5], [[3]], [7, 8, 9], 0, 16, 1), "no taken")
    got = ssq.ssq_page_fork(ints([0, 0, 0]), ints([5]), ints([[3]]), ints([]), 16, taken=ints([-4]))
    same(got, fork_reference([0, 0, 0], [5], [[3]], [], -4, 16, 1), "no free pages, an entry before the list")


POOLS = [
    # requests, longest, page, width, pages, share of pages pinned
    (1, 16, 16, 1, 1, 0), (0, 1, 16, 3, 5, 0), (3, 50, 16, 4, 0, 0), (4, 60, 16, 4, 17, 0), (5, 90, 16, 6, 40, 0.2), (64, 500, 16, 32, 4095, 0),
    (64, 500, 16, 32, 4096, 0.01), (64, 500, 16, 32, 4097, 0.01), (30, 300, 64, 5, 150, 1.0), (200, 900, 16, 60, 9000, 0.3), (7, 40, 16, 0, 30, 0),
    (300, 2000, 16, 1100, 70001, 0.001), (40, 100, 128, 1, 41, 0), (900, 700, 16, 44, 20000, 0),
]


@pytest.mark.parametrize("i", range(len(POOLS)))
def test_collect_and_compact(i):
    requests, longest, page, width, pages, share = POOLS[i]
    rng = random.Random(830 + i)
    lens = [rng.randint(-3, longest) for _ in range(requests)]
    table = [[rng.choice((-1, pages, 2 ** 31 - 1)) if rng.random() < 0.05 else rng.randrange(max(pages, 1)) for _ in range(width)] for _ in lens]
    pinned = [int(rng.random() < share) * rng.randint(1, 255) for _ in range(pages)] if share else None
    dev = [ints(lens), ints(table).view(requests, width), page, pages, None if pinned is None else torch.tensor(pinned, dtype=torch.uint8, device="cuda")]
    ws = torch.full((ssq.ssq_page_collect_workspace_size(pages, True),), 0xFF, dtype=torch.uint8, device="cuda")
    for workspace in (None, ws):
        same(ssq.ssq_page_collect(*dev, workspace=workspace), collect_reference(lens, table, page, pages, pinned), f"collect {POOLS[i]}")
        got, want = ssq.ssq_page_compact(*dev, workspace=workspace), compact_reference(lens, table, page, pages, pinned)
        same(got[1:], want[1:], f"compact {POOLS[i]}")
        assert got[0].flatten().tolist() == sum(want[0], []), f"compact {POOLS[i]}: table"
    here = [dev[1], *(torch.full_like(x, 55) for x in got[1:])]           # the table in place
    assert all(torch.equal(x, y) for x, y in zip(ssq.ssq_page_compact(*dev, out=here), got))
    out = [torch.full_like(x, 55) for x in got[1:3]]
    after = ssq.ssq_page_collect(dev[0], got[0], page, pages, pinned=dev[4], out=out)
    assert torch.equal(after[0], got[1]) and torch.equal(after[1], got[2])      # the lists after the moves


LARGE = [
    # as POOLS; past 2048 requests or 131072 pages, where marks, counts, lists and moves are launches of their own
    (2049, 40, 16, 3, 0, 0), (2049, 40, 16, 0, 30, 0.2), (2049, 20, 16, 2, 17, 0), (2049, 60, 16, 4, 4095, 0.01), (2049, 300, 16, 5, 4096, 0.4), (2049, 60, 16, 4, 4097, 0.3),
    (2500, 60, 16, 4, 9000, 0.05), (2049, 33, 16, 3, 40000, 1.0), (3000, 2000, 16, 130, 140001, 0.3), (40, 500, 16, 1030, 131073, 0.02), (1, 16, 16, 1, 131073, 0),
    # at the borders of the launch that has all marks in LDS
    (2048, 60, 16, 4, 131072, 0.1), (2048, 200, 64, 9, 131071, 0), (7, 9000, 16, 2340, 131072, 0.9),
]


@pytest.mark.parametrize("i", range(len(LARGE)))
def test_collect_and_compact_large_pools(i):
    requests, longest, page, width, pages, share = LARGE[i]
    rng = random.Random(890 + i)
    lens = [rng.randint(-3, longest) for _ in range(requests)]
    table = [[rng.choice((-1, pages, 2 ** 31 - 1)) if rng.random() < 0.05 else rng.randrange(max(pages, 1)) for _ in range(width)] for _ in lens]
    pinned = [int(rng.random() < share) * rng.randint(1, 255) for _ in range(pages)] if share else None
    check_pool(lens, table, page, pages, pinned, width, f"{LARGE[i]}")


def check_pool(lens, table, page, pages, pinned, width, tag):
    dev = [ints(lens), ints(table).view(len(lens), width), page, pages, None if pinned is None else torch.tensor(pinned, dtype=torch.uint8, device="cuda")]
    ws = torch.full((ssq.ssq_page_collect_workspace_size(pages, True) + 256,), 0xFF, dtype=torch.uint8, device="cuda")
    same(ssq.ssq_page_collect(*dev, workspace=ws[:-256]), collect_reference(lens, table, page, pages, pinned), f"collect {tag}")
    got, want = ssq.ssq_page_compact(*dev, workspace=ws[:-256]), compact_reference(lens, table, page, pages, pinned)
    assert (ws[-256:] == 0xFF).all()
    same(got[1:], want[1:], f"compact {tag}")
    assert got[0].flatten().tolist() == sum(want[0], []), f"compact {tag}: table"
    here = [dev[1].clone(), *(torch.full_like(x, 55) for x in got[1:])]           # the table in place
    assert all(torch.equal(x, y) for x, y in zip(ssq.ssq_page_compact(dev[0], here[0], *dev[2:], out=here), got)), f"in place {tag}"
    out = [torch.full_like(x, 55) for x in got[1:3]]
    after = ssq.ssq_page_collect(dev[0], got[0], page, pages, pinned=dev[4], out=out)
    assert torch.equal(after[0], got[1]) and torch.equal(after[1], got[2]), f"after the moves {tag}"


@pytest.mark.parametrize("pages", [300, 116000, 117000, 1000000, 1100000])
@pytest.mark.parametrize("compact", [False, True])
def test_outputs_do_not_keep_a_large_workspace(compact, pages):
    lens, table = ints([20, 33]), ints([[5, 9, 7], [1, 250, 2]])
    got = (ssq.ssq_page_compact if compact else ssq.ssq_page_collect)(lens, table, 16, pages)
    own = sum(x.numel() * x.element_size() for x in got)
    assert all(x.untyped_storage().nbytes() <= own + (1 << 20) + 256 for x in got)
    same(got, (compact_reference if compact else collect_reference)(lens.tolist(), table.tolist(), 16, pages), f"{pages}")


@pytest.mark.parametrize("held", [0, 1, 4095, 4096, 4097, 8192, 12288])
@pytest.mark.parametrize("pinned", [False, True])
def test_compact_where_the_held_pages_end_at_a_block(held, pinned):
    """As many held pages as whole blocks of 4096, nearly so, none and all: of a pool of three blocks, in any places."""
    pages, requests = 12288, 2051
    rng = random.Random(905 + held)
    ids = rng.sample(range(pages), held)
    width = max(1, -(-held // requests))
    table = [(ids[r * width:(r + 1) * width] + [-1] * width)[:width] for r in range(requests)]
    lens = [16 * width] * requests
    pins = None
    if pinned:                                     # of those that requests name
        pins = [0] * pages
        for e in ids[::5]:
            pins[e] = 1
    check_pool(lens, table, 16, pages, pins, width, f"{held} {pinned}")


COPIES = [
    # caches, pages, bytes a page, entries
    (1, 9, 16, 4), (2, 30, 1152, 20), (3, 12, 16400, 5), (65, 8, 4608, 4), (130, 5, 576, 2), (1, 40, 147456, 33), (2, 700, 2304, 900),
]


def test_rows_without_entries_need_no_lengths():
    """Null lens and table where the table has no columns: every page is free."""
    lib, pages = ssq.lib(), 40
    for compact in (False, True):
        need = ssq.ssq_page_collect_workspace_size(pages, compact)
        ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        free, count, src, dst, moved = (torch.full((n,), 55, dtype=torch.int32, device="cuda") for n in (pages, 1, pages // 2, pages // 2, 1))
        stream = torch.cuda.current_stream().cuda_stream
        if compact:
            st = lib.ssq_page_compact(None, 5, None, 0, 16, pages, None, None, free.data_ptr(), count.data_ptr(), src.data_ptr(), dst.data_ptr(),
                                      moved.data_ptr(), ws.data_ptr(), need, stream)
            assert moved.tolist() == [0] and set(src.tolist() + dst.tolist()) == {-1}
        else:
            st = lib.ssq_page_collect(None, 5, None, 0, 16, pages, None, free.data_ptr(), count.data_ptr(), ws.data_ptr(), need, stream)
        assert st == 0 and free.tolist() == list(range(pages)) and count.tolist() == [pages]


def test_compact_the_widest_row():
    width, pages = 2 ** 31 - 1, 100
    if torch.cuda.mem_get_info()[0] < 5 * width:
        pytest.skip("needs 10 GB of device memory")
    table = torch.full((1, width), -1, dtype=torch.int32, device="cuda")
    table[0, :4] = ints([90, 5, 99, 7])
    out = [table, *(torch.full((n,), 55, dtype=torch.int32, device="cuda") for n in (pages, 1, pages // 2, pages // 2, 1))]
    _, free, count, src, dst, moved = ssq.ssq_page_compact(ints([33]), table, 16, pages, out=out)
    assert table[0, :4].tolist() == [1, 0, 2, 7] and int(table[0, -1]) == -1       # entry 3 is behind the row's pages
    assert free.tolist() == list(range(3, 100)) + [-1] * 3 and count.tolist() == [97]
    assert src.tolist()[:4] == [5, 90, 99, -1] and dst.tolist()[:4] == [0, 1, 2, -1] and moved.tolist() == [3]


@pytest.mark.parametrize("i", range(len(COPIES)))
def test_copy(i):
    count, pages, size, entries = COPIES[i]
    g, rng = gen(850 + i), random.Random(850 + i)
    caches = [torch.randint(0, 256, (pages, size), generator=g, device="cuda", dtype=torch.uint8) for _ in range(count)]
    ids = rng.sample(range(pages), pages)
    src, dst = [-1] * entries, [-1] * entries
    for j in range(min(entries, pages // 2)):
        src[j], dst[j] = ids[2 * j], ids[2 * j + 1]
        kind = rng.randrange(8)
        if kind == 0:
            src[j] = rng.choice((-1, pages, 2 ** 31 - 1, -2 ** 31))
        elif kind == 1:
            dst[j] = rng.choice((-1, pages, 2 ** 31 - 1, -2 ** 31))
        elif kind == 2:
            dst[j] = src[j]
    order = rng.sample(range(entries), entries)
    src, dst = [src[j] for j in order], [dst[j] for j in order]
    want = [c.clone() for c in caches]
    for a, b in zip(src, dst):
        if 0 <= a < pages and 0 <= b < pages:
            for w, c in zip(want, caches):
                w[b] = c[a]
    assert ssq.ssq_page_copy(iter(caches), ints(src), ints(dst)) is None
    for j, (w, c) in enumerate(zip(want, caches)):
        assert torch.equal(w, c), f"{COPIES[i]}: cache {j}"


def test_copy_of_other_types_and_of_nothing():
    k = torch.randn((6, 2, 16, 64), device="cuda").bfloat16()
    want = k.clone()
    want[4] = k[1]
    ssq.ssq_page_copy([], ints([1]), ints([4]))
    ssq.ssq_page_copy([k], ints([]), ints([]))
    ssq.ssq_page_copy([k[:0]], ints([1]), ints([4]))
    ssq.ssq_page_copy([k, k], ints([1, -1]), ints([4, 2]))
    assert torch.equal(k, want)
    f = torch.randn((3, 1, 16, 64), device="cuda")
    want = f[2].clone()
    ssq.ssq_page_copy((f,), ints([2]), ints([0]))
    assert torch.equal(f[0], want)


def test_copy_between_far_pages():
    """Offsets beyond 2^32 bytes."""
    size = 1 << 20
    pages = (1 << 12) + 9
    cache = torch.empty((pages, size), dtype=torch.uint8, device="cuda")
    cache[0], cache[pages - 1], cache[pages - 2] = 1, 2, 3
    ssq.ssq_page_copy([cache], ints([pages - 1, 0]), ints([5, pages - 3]))
    assert (cache[5] == 2).all() and (cache[pages - 3] == 1).all() and (cache[pages - 2] == 3).all() and (cache[0] == 1).all()


# --- together, as they are used ---------------------------------------------------------------------

@pytest.mark.parametrize("kind", ["kv4", "bf16"])
def test_beams_over_a_paged_cache(kind):
    """Beams of two users: tables, stores, attention, forks with copies, users who leave, free pages collected and
    the pool compacted, step after step; every step's attention against the tokens that a beam's history holds."""
    page, hk, hq, d, users, beams = 16, 2, 4, 64, 3, 4
    rng, g = random.Random(870), gen(870)
    pages, width, n = 120, 6, users * beams
    layers = 2
    if kind == "kv4":
        caches = [ssq.ssq_kv4_cache(pages, hk, page, d) for _ in range(layers)]
    else:
        caches = [torch.zeros((pages, hk, page, d), dtype=BF, device="cuda") for _ in range(2 * layers)]
    table, lens = torch.full((n, width), -1, dtype=torch.int32, device="cuda"), ints([0] * n)
    free, count = ssq.ssq_page_collect(lens, table, page, pages)
    assert count.item() == pages
    taken = ints([0])
    history = [[] for _ in range(n)]                       # of each beam, the (k, v) rows of every layer
    for step in range(14):
        new = [rng.randint(1, 9) if step == 0 else rng.choice((1, 3)) if row or step == 0 else 0 for row in history] if step else [rng.randint(5, 20) for _ in range(n)]
        starts, lens, pos, slots, taken, _ = ssq.ssq_page_tables(lens, ints(new), free, table, page, sum(new), taken=taken)
        rows = [[A.model_like(g, (sum(new), hk, d), BF) for _ in "kv"] for _ in range(layers)]
        for layer, (k, v) in enumerate(rows):
            if kind == "kv4":
                k, v = ssq.ssq_kv4_store(k, v, slots, caches[layer], held=True)
            else:
                at = slots.long()
                caches[2 * layer][at // page, :, at % page], caches[2 * layer + 1][at // page, :, at % page] = k, v
            rows[layer] = (k, v)
        at = 0
        for r in range(n):
            history[r] = history[r] + [[(k[t], v[t]) for k, v in rows] for t in range(at, at + new[r])]
            at += new[r]
        longest = max(map(len, history))
        for layer in range(layers):
            q = A.model_like(g, (n, 1, hq, d), BF)
            if kind == "kv4":
                out = ssq.ssq_attention_decode_kv4(q, caches[layer], table, lens, longest)
                Q.check(out, *Q.decode_reference(q, caches[layer], page, table.cpu(), lens.tolist(), longest, 0), f"step {step} layer {layer}")
                k_pages, v_pages, _, _ = Q.values(caches[layer], page, d)
            else:
                out = ssq.ssq_attention_decode(q, caches[2 * layer], caches[2 * layer + 1], table, lens, longest)
                A.check(out, *A.decode_reference(q, caches[2 * layer], caches[2 * layer + 1], table.cpu(), lens.tolist(), longest, 0), f"step {step}")
                k_pages, v_pages = caches[2 * layer].cpu(), caches[2 * layer + 1].cpu()
            ids = table.cpu()
            for r in range(n):                             # the cache holds this beam's own history
                for t, token in enumerate(history[r]):
                    e = int(ids[r, t // page])
                    same_k = torch.equal(k_pages[e, :, t % page].to(BF), token[layer][0].cpu())
                    same_v = torch.equal(v_pages[e, :, t % page].to(BF), token[layer][1].cpu())
                    assert same_k and same_v, (step, r, t)
        parents = [u * beams + rng.randrange(beams) for u in range(users) for _ in range(beams)]
        if step in (6, 10):                                # a user leaves
            parents[step % 3 * beams:(step % 3 + 1) * beams] = [-1] * beams
        table, lens, src, dst, taken = ssq.ssq_page_fork(ints(parents), lens, table, free, page, taken=taken)
        ssq.ssq_page_copy(caches, src, dst)
        history = [history[p] if p >= 0 else [] for p in parents]
        assert lens.tolist() == [len(x) for x in history]
        if step % 4 == 3:
            table, free, count, src, dst, moved = ssq.ssq_page_compact(lens, table, page, pages)
            ssq.ssq_page_copy(caches, src, dst)
            taken = ints([0])
            assert count.item() + len(set(e for r, x in zip(table.tolist(), history) for e in r[:-(-len(x) // page)])) == pages
        elif step % 4 == 1:
            free, count = ssq.ssq_page_collect(lens, table, page, pages)
            taken = ints([0])


def test_fork_collect_compact_and_copy_in_a_replayed_graph():
    rng = random.Random(880)
    rows, page, pages, width = 50, 16, 600, 8
    make = lambda: ([rng.randint(0, 120) for _ in range(rows)], [rng.sample(range(pages), width) for _ in range(rows)],
                    [rng.randrange(-1, rows) for _ in range(rows)], rng.sample(range(pages), 60))
    lens, table, parents, free = make()
    dev = [ints(x) for x in (lens, table, parents, free)]
    caches = [torch.randint(0, 256, (2 * pages, 576), generator=gen(880), device="cuda", dtype=torch.uint8)]
    far = lambda x: torch.where(x >= 0, x + pages, -1)       # sources and targets apart, whatever the lists say
    def step():
        f = ssq.ssq_page_fork(dev[2], dev[0], dev[1], dev[3], page)
        c = ssq.ssq_page_collect(dev[0], dev[1], page, pages)
        m = ssq.ssq_page_compact(dev[0], dev[1], page, pages)
        ssq.ssq_page_copy(caches, m[3], far(m[4]))
        return f, c, m
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(4):
        lens, table, parents, free = make()
        for x, y in zip(dev, (lens, table, parents, free)):
            x.copy_(ints(y))
        before = caches[0].clone()
        graph.replay()
        same(out[0], fork_reference(parents, lens, table, free, 0, page, width), f"fork, replay {i}")
        same(out[1], collect_reference(lens, table, page, pages), f"collect, replay {i}")
        want = compact_reference(lens, table, page, pages)
        same(out[2], want, f"compact, replay {i}")
        for a, b in zip(want[3], want[4]):
            if a >= 0:
                before[b + pages] = before[a]
        assert torch.equal(caches[0], before), f"copy, replay {i}"
