"""Attention in 64 bits, row by row of the definition, and bounds on what the kernels may be off.

Bounds (u = 2^-24, the binary32 rounding).  With w the exact softmax weights of a row and
A = sum_j w_j |v_j| element by element:

* a score is a sum of D products in binary32: off by at most D u S, S = scale sum_d |q_d k_d|,
  and by 4 u |score| + 4 u |m| more through the scaled exponent, its reference and exp2; a weight
  is therefore off by the factor 1 + e with |e| <= eps = 2 D u max_j S_j (an exponent's error is
  its weight's relative error, and numerator and sum both carry it, so twice);
* the sums over n keys add at most 2 n u;
* bf16 (8 significant bits) rounds each weight and the output by at most 2^-8 of it.

|out - exact| <= (eps + 2 n u + 2^-20 [+ 2^-8]) A [+ 2^-8 |exact|] (the brackets in bf16); 2^-20
covers the second-order terms and the rescalings (a product each time the reference moves)."""
import math

import torch

U = 2.0 ** -24


def attend(q, k, v, last, scale):
    """(out, A, eps) of rows q [rows, d] over k, v [keys, d] in float64; row i sees keys 0..last[i]."""
    q, k, v = q.double(), k.double(), v.double()
    out = torch.zeros((q.shape[0], v.shape[1]), dtype=torch.float64, device=q.device)
    size, eps = torch.zeros_like(out), torch.zeros((q.shape[0], 1), dtype=torch.float64, device=q.device)
    for i, n in enumerate(last.tolist()):
        if n < 0:
            continue
        kk, vv = k[:n + 1], v[:n + 1]
        s = (kk * q[i]).sum(1) * scale
        w = torch.exp(s - s.max())
        w = w / w.sum()
        out[i] = (w[:, None] * vv).sum(0)
        size[i] = (w[:, None] * vv.abs()).sum(0)
        eps[i] = 2 * q.shape[1] * U * ((kk * q[i]).abs().sum(1) * scale).max() + 2 * (n + 1) * U + 2.0 ** -20
    return out, size, eps


def check(out, ref, size, eps, tag):
    bf16 = out.dtype == torch.bfloat16
    bound = (eps + (2.0 ** -8 if bf16 else 0)) * size + (2.0 ** -8 * ref.abs() if bf16 else 0)
    off = (out.double() - ref).abs()
    bad = ~(off <= bound)                         # NaN is bad too
    if bad.any():
        at = bad.nonzero()[0].tolist()
        raise AssertionError(f"{tag}: {int(bad.sum())} of {bad.numel()} off, first at {at}: got "
                             f"{out[tuple(at)].item()}, exact {ref[tuple(at)].item()}, bound {bound[tuple(at)].item()}")


def prompt_reference(q, k, v, lens, scale=None):
    scale = q.shape[2] ** -0.5 if scale is None else scale
    g = q.shape[1] // k.shape[1]
    ref, size = (torch.zeros(q.shape, dtype=torch.float64, device=q.device) for _ in range(2))
    eps = torch.zeros((*q.shape[:2], 1), dtype=torch.float64, device=q.device)
    a = 0
    for n in lens:
        last = torch.arange(n)
        for h in range(q.shape[1]):
            if n:
                ref[a:a + n, h], size[a:a + n, h], eps[a:a + n, h] = attend(q[a:a + n, h], k[a:a + n, h // g], v[a:a + n, h // g], last, scale)
        a += n
    return ref, size, eps


def gather(pages, row, row0, prefix, n, head):
    """The first n keys (or values) of a request from the paged cache, and which are present."""
    page = pages.shape[2]
    at = torch.arange(n)
    ids = torch.where(at < prefix, row0[at // page], row[at // page]) if n else at
    here = (ids >= 0) & (ids < pages.shape[0])
    return pages[ids[here].to(pages.device), head, (at[here] % page).to(pages.device)], here


def decode_reference(q, k_pages, v_pages, table, lens, max_len, prefix, scale=None):
    """As prompt_reference, for q [requests, fresh, q_heads, dim] (table, lens on the host)."""
    n, fresh, hq, d = q.shape
    scale = d ** -0.5 if scale is None else scale
    hk, page = k_pages.shape[1], k_pages.shape[2]
    g = hq // hk
    ref, size = (torch.zeros(q.shape, dtype=torch.float64, device=q.device) for _ in range(2))
    eps = torch.zeros((n, fresh, hq, 1), dtype=torch.float64, device=q.device)
    for r in range(n):
        length = max(0, min(int(lens[r]), max_len, table.shape[1] * page))
        for h in range(hk):
            k, here = gather(k_pages, table[r], table[0], prefix, length, h)
            v, _ = gather(v_pages, table[r], table[0], prefix, length, h)
            seen = torch.cumsum(here, 0) if length else here
            for i in range(fresh):
                p = length - fresh + i
                last = int(seen[p]) - 1 if p >= 0 else -1
                sl = slice(h * g, (h + 1) * g)
                ref[r, i, sl], size[r, i, sl], eps[r, i, sl] = attend(q[r, i, sl], k, v, torch.full((g,), last), scale)
    return ref, size, eps


def tables_reference(held, added, free, taken, page, table, tokens):
    """Lists of whole numbers from lists of whole numbers: starts, lens, positions, slots, taken, table."""
    starts, lens, positions, slots, table = [0], [], [], [], [list(r) for r in table]
    for r, (h, a) in enumerate(zip(held, added)):
        h, a = max(h, 0), max(a, 0)
        have, want = -(-h // page), -(-(h + a) // page)
        pages = {}
        for j in range(have, want):
            pages[j] = free[taken] if 0 <= taken < len(free) else -1
            if j < len(table[r]):
                table[r][j] = pages[j]
            taken += 1
        for t in range(h, h + a):
            j = t // page
            e = (pages[j] if j >= have else table[r][j]) if j < len(table[r]) else -1
            positions.append(t)
            slots.append(e * page + t % page if e >= 0 else -1)
        starts.append(starts[-1] + a)
        lens.append(h + a)
    pad = tokens - len(positions)
    return starts, lens, (positions + [0] * pad)[:tokens], (slots + [-1] * pad)[:tokens], taken, table


def rope_reference(x, gain, table, eps):
    """(out, bound in units of the type's half ulp is the caller's) rows [tokens, heads, d] in float64."""
    x = x.double()
    d = x.shape[2]
    if gain is not None:
        x = x / torch.sqrt((x * x).mean(2, keepdim=True) + eps) * gain.double()
    c, s = table.double()[:, None, :d // 2], table.double()[:, None, d // 2:]
    a, b = x[..., :d // 2], x[..., d // 2:]
    out = torch.cat((a * c - b * s, b * c + a * s), 2)
    size = torch.cat(((a * c).abs() + (b * s).abs(), (b * c).abs() + (a * s).abs()), 2)
    return out, size


def model_like(gen, shape, dtype, spread=0.5):
    size = (torch.randn((shape[-2], shape[-1]), generator=gen, device=gen.device) * spread).exp()
    return (torch.randn(shape, generator=gen, device=gen.device) * size).to(dtype)


def starts_of(lens):
    return [sum(lens[:i]) for i in range(len(lens) + 1)]


def pages_for(n, page):
    return math.ceil(n / page)
