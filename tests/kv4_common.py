"""The 4-bit cache by its definition (include/ssq_cache.h): bytes, values, and attention in 64 bits.

Bounds of attention over it (u = 2^-24; A, S and eps as in tests/attention_common.py, over the values that the
cache holds, which are exact: 4 bits times 11).  With c the codes and s the scales of a key:

* binary32: a query is three bf16 terms that hold its 24 bits, so that a score is a sum of 3 D exact
  products and of D / 32 scaled groups: off by at most (3 D + D / 32 + 1) u S, S = scale sum |q k|.  Weights
  times scales are three terms each too: the sums over n keys have 3 n terms, and the product that forms
  weight times scale is off by u.
* bf16: a code enters as 128 + u (at most 143), and 136 times the group's sum of q is where its sum starts; the
  start, itself a sum of 32 products, and the 32 terms are at most 64 roundings of what never exceeds 279 times
  the group's sum of |q|:  off by at most 64 * 279 u R, R = scale sum_g |s_g| sum |q_d|.
  A weight times a scale is rounded to bf16: off by 2^-8 of it at most.  For the outputs, 32 keys are 64 terms,
  at most 279 times their weights and scales in all, beside the sum itself: n keys give at most
  (64 * 279 + n / 16) u B more, B = sum_j w_j |s_j| of the element's group (the sum never exceeds 143 B).

A score's error is its weight's relative error, and numerator and sum both carry it, so eps has it twice."""
import torch

U = 2.0 ** -24
GROUP = 32


def places(page, dim):
    """Byte and shift of the code of [token, element] in a part, keys and values: [2][page, dim]."""
    g = dim // GROUP
    t, d = torch.arange(page)[:, None], torch.arange(dim)[None, :]
    grp, i = d // GROUP, d % GROUP
    keys = t * (dim // 2) + 4 * ((i // 8) * g + grp) + (i % 8) // 2
    values = (t // 4) * (2 * dim) + 4 * ((i % 16) * g + grp) + t % 4
    return [(keys, (4 * (i % 2)).expand(page, dim)), (values, (4 * (i // 16)).expand(page, dim))]


def part_bytes(page, dim):
    return page * (dim // 2 + dim // 16)


def read(cache, page, dim):
    """Codes u [pages, heads, page, dim], scales [pages, heads, page, dim / 32] of keys and of values: ((u, s), (u, s))."""
    cache = cache.cpu()
    out = []
    for which, (byte, shift) in enumerate(places(page, dim)):
        part = cache[:, :, which]
        u = (part[:, :, byte].to(torch.int32) >> shift) & 15
        s = part[:, :, page * dim // 2:].contiguous().view(torch.float16).double().unflatten(2, (page, dim // GROUP))
        out.append((u, s))
    return out


def values(cache, page, dim):
    """What the cache holds, in float64: keys, values [pages, heads, page, dim], and |scale| of each element."""
    out = []
    for u, s in read(cache, page, dim):
        by = s.repeat_interleave(GROUP, 3)
        out += [(u - 8).double() * by, by.abs()]
    return out[0], out[2], out[1], out[3]


def on_grid(x):
    """Codes u [..., dim] and scale bits (binary16, int16) [..., dim / 32] of rows x, by the definition."""
    w = x.detach().cpu().float().unflatten(-1, (-1, GROUP))
    hi, down = w.amax(-1, keepdim=True), -w.amin(-1, keepdim=True)
    most = torch.maximum(hi, down)
    s = torch.where(most > 0, torch.where(hi > down, -most, most) * torch.tensor(0.125), torch.zeros(()))        # +0 for zeros
    c = torch.where(most > 0, torch.round(w / s), torch.zeros(())).clamp(-8, 7)
    scale = s.half().squeeze(-1)
    bad = ~torch.isfinite(w).all(-1) | ~torch.isfinite(scale)
    scale = torch.where(bad, torch.tensor(float("nan"), dtype=torch.float16), scale)
    c = torch.where(bad[..., None], torch.zeros(()), c)
    return (c + 8).to(torch.int32).flatten(-2), scale


def attend(q, k, v, k_size, v_size, last, scale):
    """(out, bound) of rows q [rows, d] over the held k, v [keys, d] (|scale| of each element beside them);
    row i sees keys 0..last[i].  In float64."""
    bf16 = q.dtype == torch.bfloat16
    q, d = q.double(), q.shape[1]
    out, bound = (torch.zeros((q.shape[0], d), dtype=torch.float64) for _ in range(2))
    for i, n in enumerate(last.tolist()):
        if n < 0:
            continue
        kk, vv = k[:n + 1], v[:n + 1]
        s = (kk * q[i]).sum(1) * scale
        w = torch.exp(s - s.max())
        w = w / w.sum()
        out[i] = (w[:, None] * vv).sum(0)
        a = (w[:, None] * vv.abs()).sum(0)
        most = ((kk * q[i]).abs().sum(1) * scale).max()
        count = n + 1
        if bf16:
            reach = ((k_size[:n + 1] * q[i].abs()).sum(1) * scale).max()
            eps = 2 * (64 * 279 * U * reach + (d // 32 + 9) * U * most)
            b = (w[:, None] * v_size[:n + 1]).sum(0)
            more = (64 * 279 + count / 16) * U * b + 2.0 ** -8 * a + 2.0 ** -8 * out[i].abs()
        else:
            eps = 2 * (3 * d + d // 32 + 9) * U * most
            more = 4 * count * U * a
        bound[i] = (eps + 2 * count * U + 2.0 ** -20) * a + more
    return out, bound


def check(out, ref, bound, tag):
    off = (out.detach().cpu().double() - ref).abs()
    bad = ~(off <= bound)                         # NaN is bad too
    if bad.any():
        at = tuple(bad.nonzero()[0].tolist())
        raise AssertionError(f"{tag}: {int(bad.sum())} of {bad.numel()} off, first at {at}: got {out[at].item()}, "
                             f"exact {ref[at].item()}, bound {bound[at].item()}")


def decode_reference(q, cache, page, table, lens, max_len, prefix, scale=None):
    """(out, bound) for q [requests, fresh, q_heads, dim]; table and lens on the host."""
    q = q.detach().cpu()
    n, fresh, hq, d = q.shape
    scale = d ** -0.5 if scale is None else scale
    held = values(cache, page, d)
    pages, hk = cache.shape[:2]
    g = hq // hk
    ref, bound = (torch.zeros(q.shape, dtype=torch.float64) for _ in range(2))
    for r in range(n):
        length = max(0, min(int(lens[r]), max_len, table.shape[1] * page))
        at = torch.arange(length)
        ids = torch.where(at < prefix, table[0][at // page], table[r][at // page]) if length else at
        here = (ids >= 0) & (ids < pages)
        seen = torch.cumsum(here, 0)
        for h in range(hk):
            k, v, ks, vs = (x[ids[here].long(), h, at[here] % page] for x in held)
            for i in range(fresh):
                p = length - fresh + i
                last = int(seen[p]) - 1 if p >= 0 else -1
                sl = slice(h * g, (h + 1) * g)
                ref[r, i, sl], bound[r, i, sl] = attend(q[r, i, sl], k, v, ks, vs, torch.full((g,), last), scale)
    return ref, bound
