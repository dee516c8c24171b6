"""The attention half of a Qwen3-8B block on few-bit weights, served from a paged cache.

A system prompt is taken in once; then users join who share its pages, each with a few tokens of
their own, and are answered token by token.  Every step is

    ssq_page_tables                         once, for all layers
    ssq_matmul (q, k, v)                    the quantized projections
    ssq_qk_norm_rope                        norms and rotation, keys and values into the cache
    ssq_attention_prompt / _decode          over the prompt, or over the cache with its shared prefix
    ssq_matmul (o)

With --kv4 the cache holds 4 bits an element: ssq_kv4_store follows ssq_qk_norm_rope, the prompt attends to
its rows as the cache holds them, and ssq_attention_decode_kv4 reads them.

    python examples/attention_layer.py [--users 16] [--system 2048] [--own 4] [--tokens 32] [--kv4]
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2607_08779_amd import ssq  # noqa: E402

PAGE, GROUP, BITS = 64, 32, 4


class Layer:
    """Quantized projections, gains of the head norms, and this layer's cache."""

    def __init__(self, hidden=4096, q_heads=32, kv_heads=8, head_dim=128, pages=256, seed=0, kv4=False):
        self.hidden, self.q_heads, self.kv_heads, self.head_dim = hidden, q_heads, kv_heads, head_dim
        g = torch.Generator(device="cuda").manual_seed(seed)
        rows = {"q": q_heads * head_dim, "k": kv_heads * head_dim, "v": kv_heads * head_dim, "o": hidden}
        cols = {"q": hidden, "k": hidden, "v": hidden, "o": q_heads * head_dim}
        self.weights = {}
        for name, n in rows.items():
            w = (torch.randn((n, cols[name]), generator=g, device="cuda") * 0.02).bfloat16()
            self.weights[name] = (n, cols[name], *ssq.ssq_quantize(w, GROUP, BITS, ssq.SIGNED_SYM)[:2])
        self.q_gain, self.k_gain = ((1 + 0.1 * torch.randn(head_dim, generator=g, device="cuda")).bfloat16() for _ in "qk")
        self.pages, self.cache = pages, None
        if kv4:
            self.cache = ssq.ssq_kv4_cache(pages, kv_heads, PAGE, head_dim)
        else:
            shape = (pages, kv_heads, PAGE, head_dim)
            self.k_pages, self.v_pages = (torch.zeros(shape, dtype=torch.bfloat16, device="cuda") for _ in "kv")

    def project(self, name, x):
        n, k, codes, scales = self.weights[name]
        return ssq.ssq_matmul(x, codes, scales, None, n, k, GROUP, BITS)

    def qkv(self, x, positions, slots, rope):
        """q, k (normed, rotated) and v [tokens, heads, head_dim]; k and v are in the cache then (and, in 4 bits, what it holds)."""
        q, k, v = (self.project(n, x).view(len(x), -1, self.head_dim) for n in "qkv")
        if self.cache is not None:
            q, k = ssq.ssq_qk_norm_rope(q, k, positions, rope, q_gain=self.q_gain, k_gain=self.k_gain)
            return q, *ssq.ssq_kv4_store(k, v, slots, self.cache, held=(k, v))
        q, k = ssq.ssq_qk_norm_rope(q, k, positions, rope, q_gain=self.q_gain, k_gain=self.k_gain, v=v, slots=slots,
                                    k_pages=self.k_pages, v_pages=self.v_pages)
        return q, k, v

    def out(self, attended):
        return self.project("o", attended.view(-1, self.q_heads * self.head_dim))

    def prompt(self, x, step, rope):
        """Whole prompts, packed: x [tokens, hidden]."""
        q, k, v = self.qkv(x, step.positions, step.slots, rope)
        return self.out(ssq.ssq_attention_prompt(q, k, v, step.starts))

    def decode(self, x, fresh, step, table, max_len, prefix, rope):
        """The last `fresh` tokens of every request: x [requests * fresh, hidden]."""
        q = self.qkv(x, step.positions, step.slots, rope)[0].view(-1, fresh, self.q_heads, self.head_dim)
        if self.cache is not None:
            return self.out(ssq.ssq_attention_decode_kv4(q, self.cache, table, step.lens, max_len, prefix=prefix))
        return self.out(ssq.ssq_attention_decode(q, self.k_pages, self.v_pages, table, step.lens, max_len, prefix=prefix))


class Step:
    """Where one step's new tokens go: the same for every layer."""

    def __init__(self, held, added, tokens, free, taken, table):
        self.starts, self.lens, self.positions, self.slots, self.taken, _ = ssq.ssq_page_tables(
            held, added, free, table, PAGE, tokens, taken=taken)


def rope_table(rows, dim, theta=1e6):
    angle = torch.arange(rows, device="cuda")[:, None] * theta ** (-torch.arange(0, dim, 2, device="cuda") / dim)
    return torch.cat((angle.cos(), angle.sin()), 1)


def serve(layer, system, users, own, tokens, inputs, seen=None):
    """A system prompt of `system` tokens (whole pages), then `users` requests behind it: `own`
    tokens each at once, then `tokens` single ones.  `inputs(n)` gives n rows of activations;
    seen(kind, x, y) is told every step's input and output."""
    if system % PAGE:
        raise ValueError("shared pages have to be full")
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    max_len = system + own + tokens
    rope = rope_table(max_len, layer.head_dim)
    free = torch.arange(layer.pages, dtype=torch.int32, device="cuda")
    width = -(-max_len // PAGE)

    table = torch.full((1, width), -1, dtype=torch.int32, device="cuda")
    step = Step(i32([0]), i32([system]), system, free, i32([0]), table)
    x = inputs(system)
    y = layer.prompt(x, step, rope)
    if seen:
        seen("system", x, y)

    table = table.repeat(users, 1)                     # every user's first pages are the system prompt's
    held, taken = i32([system] * users), step.taken
    for n in [own] + [1] * tokens:
        step = Step(held, i32([n] * users), users * n, free, taken, table)
        x = inputs(users * n)
        y = layer.decode(x, n, step, table, max_len, system, rope)
        held, taken = step.lens, step.taken
        if seen:
            seen("users", x, y)
    return y


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--users", type=int, default=16)
    ap.add_argument("--system", type=int, default=2048)
    ap.add_argument("--own", type=int, default=4)
    ap.add_argument("--tokens", type=int, default=32)
    ap.add_argument("--kv4", action="store_true", help="a cache in 4 bits")
    a = ap.parse_args()
    pages = a.system // PAGE + a.users * (-(-(a.own + a.tokens) // PAGE))
    layer = Layer(pages=pages, kv4=a.kv4)
    gen = torch.Generator(device="cuda").manual_seed(1)
    inputs = lambda n: torch.randn((n, layer.hidden), generator=gen, device="cuda").bfloat16()  # noqa: E731
    serve(layer, a.system, a.users, a.own, 2, inputs)              # the first calls load and allocate
    times = []

    def seen(kind, x, y):
        torch.cuda.synchronize()
        times.append((kind, len(x), time.perf_counter()))

    torch.cuda.synchronize()
    times.append(("", 0, time.perf_counter()))
    y = serve(layer, a.system, a.users, a.own, a.tokens, inputs, seen)
    for (kind, n, t), (_, _, before) in list(zip(times[1:], times))[:4]:
        print(f"{kind}: {n} tokens in {(t - before) * 1e6:.0f} us", flush=True)
    print(f"output {tuple(y.shape)}, finite: {bool(torch.isfinite(y).all())}")


if __name__ == "__main__":
    main()
