"""Host-only checks of the attention part of the C ABI (include/ssq_attention.h): declared
symbols are exported, and invalid arguments are refused before any HIP call."""
import ctypes
import os
import re

import pytest

from paper_2607_08779_amd import ssq

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EINVAL, EALIGN = -1, -2
P = ctypes.c_void_p(1 << 20)         # aligned dummy pointers: never dereferenced, because every
OTHER = ctypes.c_void_p(1 << 21)     # call below fails validation first or has nothing to do


def off(n):
    return ctypes.c_void_p((1 << 20) + n)


NAMES = ["ssq_attention_decode", "ssq_attention_decode_f32", "ssq_attention_decode_workspace_size", "ssq_attention_prompt",
         "ssq_attention_prompt_f32", "ssq_page_tables", "ssq_qk_norm_rope", "ssq_qk_norm_rope_f32"]


def test_header_and_library_agree():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ssq_attention.h")).read(), flags=re.S)
    assert sorted(set(re.findall(r"\b(ssq_\w+)\s*\(", text))) == NAMES
    for name in NAMES:
        assert hasattr(ssq.lib(), name) and name in ssq._EXPORTS


def call(name, defaults, given):
    a = dict(defaults)
    assert set(given) <= set(a)
    a.update(given)
    return getattr(ssq.lib(), name)(*a.values())


TABLES = dict(held=P, added=P, requests=2, free_pages=P, free_count=4, taken=P, page_size=16, table=P, table_stride=3,
              tokens=5, starts=P, lens=P, positions=P, slots=P, taken_after=OTHER, stream=None)


@pytest.mark.parametrize("given", [
    dict(requests=-1), dict(requests=(1 << 20) + 1), dict(free_count=-1), dict(page_size=8), dict(page_size=48),
    dict(page_size=2048), dict(page_size=0), dict(table_stride=-1), dict(tokens=-1), dict(tokens=(1 << 30) + 1), dict(held=None),
    dict(added=None), dict(free_pages=None), dict(table=None), dict(starts=None), dict(lens=None), dict(positions=None),
    dict(slots=None), dict(taken_after=None), dict(taken=OTHER), dict(free_count=1 << 31), dict(table_stride=1 << 31),
])
def test_page_tables_refuses(given):
    assert call("ssq_page_tables", TABLES, given) == EINVAL


@pytest.mark.parametrize("which", ["held", "added", "free_pages", "taken", "table", "starts", "lens", "positions", "slots", "taken_after"])
def test_page_tables_refuses_misaligned(which):
    assert call("ssq_page_tables", TABLES, {which: off(2)}) == EALIGN


ROPE = dict(q=P, q_stride=512, k=P, k_stride=128, v=P, v_stride=128, tokens=4, q_heads=8, kv_heads=2, head_dim=64, q_gain=P,
            k_gain=P, eps=1e-6, positions=P, rope=P, rope_rows=10, q_out=P, q_out_stride=512, k_out=P, k_out_stride=128,
            slots=P, k_pages=P, v_pages=P, pages=5, page_size=16, stream=None)


@pytest.mark.parametrize("given", [
    dict(tokens=-1), dict(tokens=1 << 29), dict(q_heads=0), dict(kv_heads=0), dict(q_heads=7), dict(q_heads=1 << 17), dict(head_dim=32), dict(head_dim=96),
    dict(head_dim=256), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(rope_rows=-1), dict(q_stride=508),
    dict(q_stride=511), dict(k_stride=127), dict(v_stride=64), dict(q_out_stride=500), dict(k_out_stride=0), dict(q_stride=1 << 25),
    dict(slots=None), dict(k_pages=None), dict(v_pages=None), dict(page_size=24), dict(pages=-1), dict(pages=1 << 28), dict(q=None),
    dict(k=None), dict(v=None), dict(positions=None), dict(rope=None), dict(q_out=None), dict(q_out_stride=1024),
    dict(k_out=None, slots=None, k_pages=None, v_pages=None), dict(k_out_stride=256),
])
def test_norm_rope_refuses(given):
    for name in ("ssq_qk_norm_rope", "ssq_qk_norm_rope_f32"):
        assert call(name, ROPE, given) == EINVAL


@pytest.mark.parametrize("which", ["q", "k", "v", "q_gain", "k_gain", "rope", "q_out", "k_out", "k_pages", "v_pages"])
def test_norm_rope_refuses_misaligned(which):
    for name in ("ssq_qk_norm_rope", "ssq_qk_norm_rope_f32"):
        assert call(name, ROPE, {which: off(8)}) == EALIGN
        assert call(name, ROPE, {"positions": off(2)}) == EALIGN and call(name, ROPE, {"slots": off(1)}) == EALIGN
    assert call("ssq_qk_norm_rope", ROPE, dict(q_stride=516)) == EINVAL       # not a multiple of 16 bytes


PROMPT = dict(q=P, q_stride=512, k=P, k_stride=128, v=P, v_stride=128, starts=P, requests=2, tokens=40, q_heads=8, kv_heads=2,
              head_dim=64, scale=0.125, out=OTHER, out_stride=512, stream=None)


@pytest.mark.parametrize("given", [
    dict(requests=-1), dict(requests=1 << 21), dict(tokens=-1), dict(tokens=1 << 28), dict(q_heads=0), dict(kv_heads=3), dict(kv_heads=0),
    dict(head_dim=80), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(q_stride=256),
    dict(k_stride=120), dict(v_stride=130), dict(out_stride=510), dict(k_stride=(1 << 24) + 8), dict(q=None), dict(k=None), dict(v=None),
    dict(starts=None), dict(out=None), dict(requests=1 << 20, q_heads=1 << 12, kv_heads=1 << 10, q_stride=1 << 18),
])
def test_prompt_refuses(given):
    for name in ("ssq_attention_prompt", "ssq_attention_prompt_f32"):
        assert call(name, PROMPT, given) == EINVAL


@pytest.mark.parametrize("which,by", [("q", 8), ("k", 4), ("v", 2), ("out", 8), ("starts", 2)])
def test_prompt_refuses_misaligned(which, by):
    for name in ("ssq_attention_prompt", "ssq_attention_prompt_f32"):
        assert call(name, PROMPT, {which: off(by)}) == EALIGN


DECODE = dict(q=P, q_stride=512, requests=3, fresh=2, q_heads=8, kv_heads=2, head_dim=64, scale=0.125, k_pages=P, v_pages=P, pages=9,
              page_size=16, table=P, table_stride=4, lens=P, max_len=50, prefix=20, out=OTHER, out_stride=512, workspace=P,
              workspace_bytes=0, stream=None)


@pytest.mark.parametrize("given", [
    dict(requests=-1), dict(requests=1 << 21), dict(fresh=0), dict(fresh=-3), dict(fresh=1 << 30), dict(q_heads=9), dict(kv_heads=0),
    dict(head_dim=100), dict(scale=0.0), dict(scale=float("nan")), dict(pages=-1), dict(pages=1 << 27), dict(page_size=17), dict(page_size=8),
    dict(table_stride=-1), dict(max_len=-1), dict(max_len=(1 << 30) + 1), dict(prefix=-1), dict(q_stride=511), dict(out_stride=256),
    dict(q=None), dict(out=None), dict(lens=None), dict(table=None), dict(k_pages=None), dict(v_pages=None),
])
def test_decode_refuses(given):
    for name in ("ssq_attention_decode", "ssq_attention_decode_f32"):
        assert call(name, DECODE, given) == EINVAL


@pytest.mark.parametrize("which,by", [("q", 8), ("k_pages", 8), ("v_pages", 4), ("out", 8), ("table", 2), ("lens", 1), ("workspace", 128)])
def test_decode_refuses_misaligned(which, by):
    for name in ("ssq_attention_decode", "ssq_attention_decode_f32"):
        assert call(name, DECODE, {which: off(by)}) == EALIGN


def test_nothing_to_do():
    assert call("ssq_qk_norm_rope", ROPE, dict(tokens=0, q=None, k=None)) == 0
    assert call("ssq_attention_prompt", PROMPT, dict(tokens=0, q=None)) == 0
    assert call("ssq_attention_decode", DECODE, dict(requests=0, q=None)) == 0


def test_decode_workspace_sizes():
    size = ssq.ssq_attention_decode_workspace_size
    assert size(0, 1, 32, 8, 128, 1000) == 0 and size(1, 1, 32, 8, 100, 1000) == 0 and size(-1, 1, 32, 8, 128, 1000) == 0
    assert size(1, 1, 32, 8, 128, 16) == 0                                     # nothing to split
    long = size(1, 1, 32, 8, 128, 16384)
    assert long > 0 and long % (32 * (8 + 4 * 128)) == 0                       # whole parts: m, l and D values a row
    assert size(1, 1, 32, 8, 128, 16384, 8192) == long                         # one request shares nothing
    assert size(64, 1, 32, 8, 128, 9000, 8192) > 0
