"""Host-only checks of the third part of the C ABI (include/ssq_cache.h): declared symbols are exported, and invalid
arguments are refused before any HIP call; and the Python binding's own checks, on host tensors."""
import ctypes
import os
import re

import pytest
import torch

from paper_2607_08779_amd import ssq
from tests.test_attention_host import EALIGN, EINVAL, ROOT, call, off
from tests.test_attention_binding import reaches_the_library

NAMES = ["ssq_attention_decode_kv4", "ssq_attention_decode_kv4_f32", "ssq_attention_decode_kv4_workspace_size", "ssq_kv4_store", "ssq_kv4_store_f32",
         "ssq_page_collect", "ssq_page_collect_workspace_size", "ssq_page_compact", "ssq_page_copy", "ssq_page_fork"]


def at(i):
    """Pointers 1 MiB apart that are never dereferenced."""
    return off(i << 20)


def test_header_and_library_agree():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ssq_cache.h")).read(), flags=re.S)
    assert sorted(set(re.findall(r"\b(ssq_\w+)\s*\(", text))) == NAMES
    for name in NAMES:
        assert hasattr(ssq.lib(), name) and name in ssq._EXPORTS


STORE = dict(k=at(0), k_stride=128, v=at(1), v_stride=128, tokens=4, kv_heads=2, head_dim=64, slots=at(2), cache=at(3), pages=5, page_size=16, k_held=at(4),
             k_held_stride=128, v_held=at(5), v_held_stride=128, stream=None)


@pytest.mark.parametrize("given", [
    dict(tokens=-1), dict(tokens=(1 << 30) + 1), dict(kv_heads=0), dict(kv_heads=1 << 17), dict(head_dim=32), dict(head_dim=96), dict(head_dim=256), dict(page_size=8),
    dict(page_size=48), dict(page_size=2048), dict(pages=-1), dict(pages=1 << 27), dict(k_stride=127), dict(k_stride=64), dict(v_stride=132), dict(k_stride=1 << 25),
    dict(k_held_stride=120), dict(v_held_stride=0), dict(k=None), dict(v=None), dict(slots=None), dict(cache=None), dict(k_held=at(0), k_held_stride=256),
    dict(v_held=at(1), v_held_stride=256), dict(tokens=1 << 29, kv_heads=2),
])
def test_store_refuses(given):
    for name in ("ssq_kv4_store", "ssq_kv4_store_f32"):
        if given.get("v_stride") == 132 and name.endswith("f32"):
            continue                                                      # whole 16 bytes in binary32
        assert call(name, STORE, given) == EINVAL, (name, given)


@pytest.mark.parametrize("which,n", [("k", 8), ("v", 4), ("cache", 8), ("k_held", 2), ("v_held", 8), ("slots", 2)])
def test_store_refuses_misaligned(which, n):
    for name in ("ssq_kv4_store", "ssq_kv4_store_f32"):
        assert call(name, STORE, {which: off(((9 << 20)) + n)}) == EALIGN
        assert call(name, STORE, {"tokens": 0, which: off((9 << 20) + n)}) == 0


def test_store_refuses_what_no_launch_holds():
    """A workgroup for 16 tokens of a head of 128, 32 of a head of 64, fewer than 2^24 of them."""
    given = dict(kv_heads=16, head_dim=128, k_stride=2048, v_stride=2048, k_held=None, v_held=None, k=off(8))
    assert call("ssq_kv4_store", STORE, {**given, "tokens": (1 << 24) - 15}) == EINVAL
    assert call("ssq_kv4_store", STORE, {**given, "tokens": (1 << 24) - 16}) == EALIGN
    assert call("ssq_kv4_store", STORE, {**given, "head_dim": 64, "tokens": (1 << 25) - 31}) == EINVAL
    assert call("ssq_kv4_store", STORE, {**given, "head_dim": 64, "tokens": (1 << 25) - 32}) == EALIGN


K_AT, ROW, CACHE_BYTES = at(0).value, 2 * 64 * 2, 5 * 2 * 2 * 16 * 36            # of STORE: 4 rows of 256 bytes, the cache


@pytest.mark.parametrize("given", [
    # written rows over rows that are read: moved by a part of a row, by whole rows, in other strides, between the rows and reaching into them
    dict(k_held=off(16)), dict(k_held=off(ROW)), dict(k_held=off(-3 * ROW)), dict(v_held=off(1 << 20), v_held_stride=136), dict(k_held=at(1)), dict(v_held=at(0)),
    dict(k_stride=384, k_held=off(1536 + 240), k_held_stride=384), dict(k_stride=1024, k_held=off(ROW), k_held_stride=680), dict(k_held=off(3 * ROW + 240)),
    dict(k=at(1), v=at(1), k_held=at(1), v_held=off((1 << 20) + 16)),
    # the two outputs
    dict(v_held=at(4)), dict(v_held=off((4 << 20) + 16)), dict(k_stride=384, v_stride=384, k_held_stride=384, v_held_stride=384, v_held=off((4 << 20) + 240)),
    dict(k=at(1), v=at(1), k_held=at(4), v_held=at(4), v_held_stride=256),
    # the cache and the slots
    dict(cache=at(0)), dict(cache=off((1 << 20) + 3 * ROW)), dict(cache=at(4)), dict(cache=off((5 << 20) - CACHE_BYTES + 16)), dict(slots=off((3 << 20) + 32)),
    dict(slots=off((3 << 20) - 12)), dict(slots=off((4 << 20) + 60)), dict(slots=off((5 << 20) - 4)), dict(slots=off((3 << 20) + CACHE_BYTES - 4)),
])
def test_store_refuses_outputs_over_other_arrays(given):
    assert call("ssq_kv4_store", STORE, given) == EINVAL == call("ssq_kv4_store_f32", STORE, given), given


DECODE = dict(q=at(0), q_stride=512, requests=2, fresh=1, q_heads=8, kv_heads=2, head_dim=64, scale=0.125, cache=at(1), pages=5, page_size=16, table=at(2),
              table_stride=3, lens=at(3), max_len=40, prefix=0, out=at(4), out_stride=512, workspace=None, workspace_bytes=0, stream=None)


@pytest.mark.parametrize("given", [
    dict(requests=-1), dict(requests=(1 << 20) + 1), dict(fresh=0), dict(q_heads=7), dict(kv_heads=0), dict(head_dim=80), dict(scale=0.0), dict(scale=-1.0),
    dict(scale=float("nan")), dict(scale=float("inf")), dict(pages=-1), dict(pages=1 << 27), dict(page_size=20), dict(table_stride=-1), dict(table_stride=1 << 31),
    dict(max_len=-1), dict(max_len=(1 << 30) + 1), dict(prefix=-1), dict(q_stride=500), dict(q_stride=508), dict(out_stride=0), dict(q=None), dict(out=None),
    dict(lens=None), dict(table=None), dict(cache=None), dict(requests=1 << 20, q_heads=16, kv_heads=8, fresh=8),
])
def test_decode_refuses(given):
    for name in ("ssq_attention_decode_kv4", "ssq_attention_decode_kv4_f32"):
        assert call(name, DECODE, given) == EINVAL, (name, given)


@pytest.mark.parametrize("which,n", [("q", 8), ("cache", 8), ("out", 8), ("table", 2), ("lens", 1), ("workspace", 128)])
def test_decode_refuses_misaligned(which, n):
    for name in ("ssq_attention_decode_kv4", "ssq_attention_decode_kv4_f32"):
        assert call(name, DECODE, {which: off((9 << 20) + n)}) == EALIGN
        assert call(name, DECODE, {"requests": 0, which: off((9 << 20) + n)}) == 0


def test_decode_refuses_what_no_launch_holds():
    """ceil(fresh * group / 16) workgroups a request and key/value head, fewer than 2^24."""
    wide = dict(q_stride=1 << 11, out_stride=1 << 11, q=off(8), fresh=1)
    assert call("ssq_attention_decode_kv4", DECODE, {**wide, "requests": 1 << 20, "q_heads": 15, "kv_heads": 15}) == EALIGN
    assert call("ssq_attention_decode_kv4", DECODE, {**wide, "requests": 1 << 20, "q_heads": 16, "kv_heads": 16}) == EINVAL
    assert call("ssq_attention_decode_kv4", DECODE, {**wide, "requests": 1, "fresh": (1 << 24) - 1, "q_heads": 16, "kv_heads": 1}) == EINVAL
    assert call("ssq_attention_decode_kv4", DECODE, {**wide, "requests": 1, "fresh": (1 << 24) - 2, "q_heads": 16, "kv_heads": 1}) == EALIGN
    size = ssq.ssq_attention_decode_kv4_workspace_size
    assert size(2, 1, 8, 2, 64, 40) == size(2, 1, 8, 2, 96, 40000) == size(0, 1, 8, 2, 64, 4000) == 0 < size(2, 1, 8, 2, 64, 4000)
    assert size(1 << 20, 1, 16, 16, 64, 4096, 2048) == 0


FORK = dict(parents=at(0), requests=3, lens=at(1), table=at(2), rows=2, table_stride=4, free_pages=at(3), free_count=5, taken=at(4), page_size=16,
            table_out=at(5), table_out_stride=4, lens_out=at(6), src=at(7), dst=at(8), taken_after=at(9), stream=None)


@pytest.mark.parametrize("given", [
    dict(requests=-1), dict(requests=(1 << 14) + 1), dict(rows=-1), dict(rows=(1 << 14) + 1), dict(table_stride=-1), dict(table_stride=1 << 31),
    dict(table_out_stride=-1), dict(table_out_stride=1 << 31), dict(free_count=-1), dict(free_count=1 << 31), dict(page_size=24), dict(parents=None), dict(lens=None),
    dict(table=None), dict(free_pages=None), dict(table_out=None), dict(lens_out=None), dict(src=None), dict(dst=None), dict(taken_after=None),
])
def test_fork_refuses(given):
    assert call("ssq_page_fork", FORK, given) == EINVAL


FORK_COUNT = dict(parents=3, lens=2, table=8, free_pages=5, taken=1, table_out=12, lens_out=3, src=3, dst=3, taken_after=1)


@pytest.mark.parametrize("written", ["table_out", "lens_out", "src", "dst", "taken_after"])
@pytest.mark.parametrize("other", list(FORK_COUNT))
def test_fork_refuses_outputs_over_other_arrays(written, other):
    start = FORK[other].value
    for first in {start, start + 4 * (FORK_COUNT[other] - 1), start - 4 * (FORK_COUNT[written] - 1)} if other != written else ():
        assert call("ssq_page_fork", FORK, {written: ctypes.c_void_p(first)}) == EINVAL, (written, other)
    assert call("ssq_page_fork", FORK, {other: off((50 << 20) + 2)}) == EALIGN


COLLECT = dict(lens=at(0), requests=2, table=at(1), table_stride=4, page_size=16, pages=10, pinned=at(2), free_pages=at(3), count=at(4), workspace=at(5),
               workspace_bytes=1 << 19, stream=None)
COMPACT = dict(lens=at(0), requests=2, table=at(1), table_stride=4, page_size=16, pages=10, pinned=at(2), table_out=at(6), free_pages=at(3), count=at(4),
               src=at(7), dst=at(8), moved=at(9), workspace=at(5), workspace_bytes=1 << 19, stream=None)


@pytest.mark.parametrize("given", [
    dict(requests=-1), dict(requests=(1 << 20) + 1), dict(table_stride=-1), dict(table_stride=1 << 31), dict(page_size=0), dict(pages=-1), dict(pages=1 << 27),
    dict(lens=None), dict(table=None), dict(free_pages=None), dict(count=None), dict(workspace=None), dict(workspace_bytes=100), dict(requests=1 << 14, table_stride=1 << 20),
])
def test_collect_and_compact_refuse(given):
    assert call("ssq_page_collect", COLLECT, given) == EINVAL and call("ssq_page_compact", COMPACT, given) == EINVAL


def test_compact_refuses():
    for which in ("table_out", "src", "dst", "moved"):
        assert call("ssq_page_compact", COMPACT, {which: None}) == EINVAL


POOL_BYTES = dict(lens=8, table=32, pinned=10, free_pages=40, count=4, table_out=32, src=20, dst=20, moved=4, workspace=1 << 19)


@pytest.mark.parametrize("written", ["table_out", "free_pages", "count", "src", "dst", "moved", "workspace"])
@pytest.mark.parametrize("other", list(POOL_BYTES))
def test_collect_and_compact_refuse_outputs_over_other_arrays(written, other):
    for name, defaults in (("ssq_page_collect", COLLECT), ("ssq_page_compact", COMPACT)):
        if written not in defaults or other not in defaults or other == written:
            continue
        start = defaults[other].value
        for first in {start, start + POOL_BYTES[other] - 4, start - POOL_BYTES[written] + (256 if written == "workspace" else 4)}:
            if {written, other} == {"table", "table_out"} and first == start:
                continue                                                  # in place
            first = first & ~255 if written == "workspace" else first & ~3
            assert call(name, defaults, {written: ctypes.c_void_p(first)}) == EINVAL, (name, written, other)
    for which, n in (("lens", 2), ("table", 1), ("free_pages", 2), ("count", 2), ("workspace", 128)):
        assert call("ssq_page_collect", COLLECT, {which: off((50 << 20) + n)}) == EALIGN == call("ssq_page_compact", COMPACT, {which: off((50 << 20) + n)})


@pytest.mark.parametrize("other", ["lens", "pinned", "free_pages", "count", "src", "dst", "moved", "workspace"])
def test_compact_in_place_refuses_other_arrays_in_the_table(other):
    """Where the table is renamed in place, it is written while other workgroups still read lengths and pins."""
    here, size = COMPACT["table"].value, POOL_BYTES[other]
    for first in (here, here - size + 256) if other == "workspace" else (here, here + 16, here + POOL_BYTES["table"] - 4, here - size + 4 & ~3):
        assert call("ssq_page_compact", COMPACT, {"table_out": COMPACT["table"], other: ctypes.c_void_p(first)}) == EINVAL, (other, first)


def copy(caches, page_bytes=1152, pages=5, src=at(20), dst=at(21), entries=3, count=None):
    pointers = (ctypes.c_void_p * max(len(caches), 1))(*(c.value if c else None for c in caches)) if caches is not None else None
    return ssq.lib().ssq_page_copy(pointers, len(caches or ()) if count is None else count, page_bytes, pages, src, dst, entries, None)


def test_copy_refuses():
    assert copy([at(0), None]) == copy(None, count=2) == copy([at(0)], src=None) == copy([at(0)], dst=None) == EINVAL
    for bad in (dict(page_bytes=0), dict(page_bytes=-16), dict(page_bytes=1160), dict(page_bytes=(1 << 30) + 16), dict(pages=-1), dict(pages=1 << 31), dict(entries=-1),
                dict(entries=(1 << 30) + 1), dict(count=-1), dict(count=(1 << 16) + 1)):
        assert copy([at(0)], **bad) == EINVAL, bad
    assert copy([at(0), off(8)]) == copy([at(0)], src=off(2)) == copy([at(0)], dst=off(1)) == EALIGN
    assert copy([]) == copy([at(0)], entries=0) == copy([at(0)], pages=0) == 0
    for over in (dict(src=off(5 * 1152 - 4)), dict(dst=off(16))):                    # lists inside a cache
        assert copy([at(3), at(0)], **over) == EINVAL


# --- the binding ---------------------------------------------------------------------------------

BF = torch.bfloat16


def test_binding_of_the_store():
    k = torch.zeros((5, 2, 64), dtype=BF)
    cache, slots = torch.zeros((3, 2, 2, 16 * 36), dtype=torch.uint8), torch.zeros(5, dtype=torch.int32)
    reaches_the_library(lambda: ssq.ssq_kv4_store(k, k, slots, cache))
    reaches_the_library(lambda: ssq.ssq_kv4_store(k, k, slots, cache, held=(k, k)))
    for bad in (lambda: ssq.ssq_kv4_store(k, k[:4], slots, cache), lambda: ssq.ssq_kv4_store(k, k[:, :1], slots, cache), lambda: ssq.ssq_kv4_store(k, k.float(), slots, cache),
                lambda: ssq.ssq_kv4_store(k, k, slots, cache[:, :1]), lambda: ssq.ssq_kv4_store(k, k, slots, cache[..., :-4]), lambda: ssq.ssq_kv4_store(k, k, slots, cache[:, :, :1]),
                lambda: ssq.ssq_kv4_store(k, k, slots, cache, held=(k, k[:4])), lambda: ssq.ssq_kv4_store(k.transpose(1, 2), k, slots, cache),
                lambda: ssq.ssq_kv4_store(k, k, slots, cache.view(torch.int8))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        ssq.ssq_kv4_store(k.half(), k.half(), slots, cache)


def test_binding_of_decoding():
    q, cache = torch.zeros((2, 1, 8, 64), dtype=BF), torch.zeros((4, 2, 2, 16 * 36), dtype=torch.uint8)
    table, lens = torch.zeros((2, 2), dtype=torch.int32), torch.ones(2, dtype=torch.int32)
    reaches_the_library(lambda: ssq.ssq_attention_decode_kv4(q, cache, table, lens, 32, workspace=torch.empty(8, dtype=torch.uint8)))
    for bad in (torch.empty(1, dtype=torch.uint8).expand(1 << 20), torch.empty(1 << 21, dtype=torch.uint8)[::2]):
        with pytest.raises(ValueError):
            ssq.ssq_attention_decode_kv4(q, cache, table, lens, 32, workspace=bad)
    for bad in (lambda: ssq.ssq_attention_decode_kv4(q[0], cache, table, lens, 32), lambda: ssq.ssq_attention_decode_kv4(q, cache[0], table, lens, 32),
                lambda: ssq.ssq_attention_decode_kv4(q, cache[..., :100], table, lens, 32), lambda: ssq.ssq_attention_decode_kv4(q, cache, table[0], lens, 32),
                lambda: ssq.ssq_attention_decode_kv4(q, cache, table, lens, 32, out=q.float())):
        with pytest.raises(ValueError):
            bad()


def test_binding_of_pages():
    i = lambda *shape: torch.zeros(shape, dtype=torch.int32)
    for bad in (lambda: ssq.ssq_page_fork(i(2, 1), i(2), i(2, 3), i(4), 16), lambda: ssq.ssq_page_fork(i(2), i(2), i(3), i(4), 16),
                lambda: ssq.ssq_page_fork(i(2), i(2), i(2, 3), i(4), 16, width=-1), lambda: ssq.ssq_page_fork(i(2), i(3), i(2, 3), i(4), 16),
                lambda: ssq.ssq_page_fork(i(2), i(2), i(2, 3), i(4), 16, out=(i(2, 4), i(2), i(2), i(2), i(1)), width=5), lambda: ssq.ssq_page_collect(i(2, 1), i(2, 3), 16, 5),
                lambda: ssq.ssq_page_collect(i(2), i(2), 16, 5), lambda: ssq.ssq_page_collect(i(2), i(2, 3), 16, -1), lambda: ssq.ssq_page_compact(i(2), i(2, 3), 16, -5),
                lambda: ssq.ssq_page_copy([i(4, 4), i(5, 4)], i(1), i(1)), lambda: ssq.ssq_page_copy([i(4, 4), i(4, 8)], i(1), i(1)),
                lambda: ssq.ssq_page_copy([i(4, 8)[:, ::2]], i(1), i(1)), lambda: ssq.ssq_page_copy([i(4, 4)], i(1, 1), i(1)), lambda: ssq.ssq_page_copy([torch.zeros(())], i(1), i(1))):
        with pytest.raises(ValueError):
            bad()
    reaches_the_library(lambda: ssq.ssq_page_copy([i(4, 4), i(4, 2, 2)], i(1), i(1)))
    reaches_the_library(lambda: ssq.ssq_page_collect(i(2), i(2, 3), 16, 5, workspace=torch.empty(8, dtype=torch.uint8)))
