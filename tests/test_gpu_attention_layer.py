"""examples/attention_layer.py against the layer's definition: every step's attention in 64 bits
over all tokens so far, on the outputs of the layer's own projections."""
import importlib.util
import os

import pytest
import torch

from tests import attention_common as A

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("attention_layer", os.path.join(ROOT, "examples", "attention_layer.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_layer_serves_users_behind_a_system_prompt():
    ex = example()
    system, users, own, tokens = 128, 5, 3, 4
    hq, hk, d = 8, 2, 64
    layer = ex.Layer(hidden=256, q_heads=hq, kv_heads=hk, head_dim=d, pages=system // ex.PAGE + users, seed=3)
    gen = torch.Generator(device="cuda").manual_seed(4)
    steps = []
    ex.serve(layer, system, users, own, tokens, lambda n: torch.randn((n, 256), generator=gen, device="cuda").bfloat16(),
             lambda kind, x, y: steps.append((x, y)))
    rope = ex.rope_table(system + own + tokens, d)

    def heads(x, positions):
        """q, k as the cache holds them (bf16), and v."""
        q, k, v = (layer.project(n, x).view(len(x), -1, d) for n in "qkv")
        q, k = (A.rope_reference(t, g, rope[positions], 1e-6)[0].bfloat16() for t, g in ((q, layer.q_gain), (k, layer.k_gain)))
        return q, k, v

    def near(y, attended):
        """The o projection of the definition's rows: what bf16 rounding of q, k, the weights and the
        rows puts between the two is a few 2^-8 of the rows, and so of their products."""
        want = layer.out(attended.bfloat16().reshape(len(y), -1)).double()
        assert (y.double() - want).norm() <= 6 * 2.0 ** -8 * want.norm()

    x, y = steps[0]
    q, k0, v0 = heads(x, torch.arange(system, device="cuda"))
    near(y, A.prompt_reference(q, k0, v0, [system])[0])
    past = [(k0, v0)] * users
    at = system
    for x, y in steps[1:]:
        n = len(x) // users
        positions = torch.arange(at, at + n, device="cuda").repeat(users)
        q, k, v = heads(x, positions)
        rows = []
        for r in range(users):
            own_rows = slice(r * n, r * n + n)
            past[r] = torch.cat((past[r][0], k[own_rows])), torch.cat((past[r][1], v[own_rows]))
            last = torch.arange(at, at + n)
            rows.append(torch.stack([A.attend(q[own_rows, h], past[r][0][:, h * hk // hq], past[r][1][:, h * hk // hq], last, d ** -0.5)[0]
                                     for h in range(hq)], 1))
        near(y, torch.cat(rows))
        at += n
    assert at == system + own + tokens and len(steps) == 2 + tokens


def test_layer_refuses_a_shared_page_that_is_not_full():
    ex = example()
    layer = ex.Layer(hidden=128, q_heads=2, kv_heads=1, head_dim=64, pages=4)
    with pytest.raises(ValueError):
        ex.serve(layer, 100, 2, 1, 1, lambda n: torch.zeros((n, 128), device="cuda").bfloat16())
