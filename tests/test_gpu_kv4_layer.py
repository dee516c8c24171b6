"""examples/attention_layer.py on a cache in 4 bits against the layer's definition: every step's attention in 64
bits over what the grid holds of all tokens so far, on the outputs of the layer's own projections."""
import pytest
import torch

from tests import attention_common as A
from tests import kv4_common as Q
from tests.test_gpu_attention_layer import example

pytestmark = pytest.mark.gpu


def held(x):
    u, scale = Q.on_grid(x)
    return ((u - 8).double() * scale.double().repeat_interleave(32, 2)).cuda()


def test_layer_serves_users_from_a_cache_in_4_bits():
    ex = example()
    system, users, own, tokens = 128, 4, 3, 3
    hq, hk, d = 8, 2, 64
    layer = ex.Layer(hidden=256, q_heads=hq, kv_heads=hk, head_dim=d, pages=system // ex.PAGE + users, seed=5, kv4=True)
    gen = torch.Generator(device="cuda").manual_seed(6)
    steps = []
    ex.serve(layer, system, users, own, tokens, lambda n: torch.randn((n, 256), generator=gen, device="cuda").bfloat16(),
             lambda kind, x, y: steps.append((x, y)))
    rope = ex.rope_table(system + own + tokens, d)

    def heads(x, positions):
        q, k, v = (layer.project(n, x).view(len(x), -1, d) for n in "qkv")
        q, k = (A.rope_reference(t, g, rope[positions], 1e-6)[0].bfloat16() for t, g in ((q, layer.q_gain), (k, layer.k_gain)))
        return q, held(k), held(v)

    def near(y, attended):
        """The o projection of the definition's rows: bf16 rounding of q, the weights, the values as the prompt
        reads them and the rows puts a few 2^-8 of the rows between the two, as in the layer on bf16.  A key that
        binary32 and 64 bits round to different sides changes a code in some 2^-18 of the elements, by an eighth of
        the group's largest: 2^-10 of the rows at most."""
        want = layer.out(attended.bfloat16().reshape(len(y), -1)).double()
        assert (y.double() - want).norm() <= 7 * 2.0 ** -8 * want.norm()

    x, y = steps[0]
    q, k0, v0 = heads(x, torch.arange(system, device="cuda"))
    near(y, A.prompt_reference(q, k0.bfloat16(), v0.bfloat16(), [system])[0])
    past = [(k0, v0)] * users
    at = system
    for x, y in steps[1:]:
        n = len(x) // users
        q, k, v = heads(x, torch.arange(at, at + n, device="cuda").repeat(users))
        rows = []
        for r in range(users):
            mine = slice(r * n, r * n + n)
            past[r] = torch.cat((past[r][0], k[mine])), torch.cat((past[r][1], v[mine]))
            last = torch.arange(at, at + n)
            rows.append(torch.stack([A.attend(q[mine, h], past[r][0][:, h * hk // hq], past[r][1][:, h * hk // hq], last, d ** -0.5)[0] for h in range(hq)], 1))
        near(y, torch.cat(rows))
        at += n
    assert at == system + own + tokens and len(steps) == 2 + tokens
