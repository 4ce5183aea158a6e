"""Prompt attention where one key's score lies far above all others, at every place of a step, against fp64."""
import pytest
import torch

from operator_refs import SlabPool, within
from prompt_refs import append_new, call_prefill, prefill_reference, up16

pytestmark = pytest.mark.gpu

LONG = 128.0        # of a query's vector: scores of ordinary keys are about 1 in size


def one_far_key(kind, q_heads, hkv, d, ctx, new, places, jump, ctas):
    """places[i * hkv + h]: the position of the key of request i and KV head h whose scaled score is `jump` above the others'."""
    n = len(places) // hkv
    s = SlabPool([up16(ctx + new)] * n, [ctx] * n, 1, hkv, d, kind, seed=int(jump), ctas=ctas, max_batch=n)
    t = s.tables(list(range(n)), [new] * n)
    append_new(s, t, 0, [new] * n)
    u = torch.ones(d) / d ** 0.5
    keys = 0.1 * torch.randn(n, hkv, ctx + new, d, generator=s.gen)
    for i, at in enumerate(places):
        keys[i // hkv, i % hkv, at] = u * (jump * d ** 0.5 / LONG)
    for i in range(n):
        for h in range(hkv):
            row = s.base[i] * hkv + h * s.caps[i]
            s.mem[0, row:row + ctx + new] = s.stored(keys[i, h], 0).cuda()
    q = (u * LONG).expand(n * new, q_heads, d).to(s.io).cuda().contiguous()
    out, lse = call_prefill(s, 0, q, t)
    want = prefill_reference(s, 0, q, list(range(n)), [ctx] * n, [new] * n, twice=True)
    # Weights are fp32 numbers against a reference that is no higher than the largest score, so their sum is at least 1.  Ordinary
    # keys' are below 2^-126 here, the least normal number: each may be 0 or anything below 2^-125 instead, which moves the
    # result by at most 2^-125 times the sum of |v|.  (It shows where the far key's own value is 0.)
    size = torch.stack([torch.stack([s.values(1, r, h, ctx + new).abs().sum(0) for h in range(hkv)]) for r in range(n)])
    under = 2.0 ** -125 * size.repeat_interleave(q_heads // hkv, 1).repeat_interleave(new, 0)
    within(out, want[0], want[2] + under, "out")
    within(lse, want[1], want[3], "lse")


# in powers of two 127, 128.4, 130, 144, 202, 289, 369, 433, 635 and 1,010
JUMPS = [88.1, 89.0, 90.1, 100.0, 140.0, 200.0, 256.0, 300.0, 440.0, 700.0]


@pytest.mark.parametrize("kind,q_heads,d", [("bf16", 28, 128), ("bf16", 16, 64), ("e4m3", 28, 128), ("f32", 8, 64)])
@pytest.mark.parametrize("ctas", [1, 37, 148])
@pytest.mark.parametrize("jump", JUMPS)
def test_one_key_far_above_all_others(kind, q_heads, d, ctas, jump):
    """At every place of the second step of 128 keys, which every token sees whole, and at the first and last places around it."""
    one_far_key(kind, q_heads, 4, d, 400, 3, list(range(128, 256)), jump, ctas)
    one_far_key(kind, q_heads, 4, d, 400, 3, [0, 127, 256, 266, 383, 384, 394, 399], jump, ctas)


@pytest.mark.parametrize("kind,q_heads,d", [("bf16", 28, 128), ("bf16", 16, 64), ("e4m3", 28, 128), ("f32", 8, 64)])
@pytest.mark.parametrize("jump", [90.1, 300.0])
def test_one_key_far_above_all_others_of_a_cut_tile(kind, q_heads, d, jump):
    """One request, its tile cut into many pieces: every piece has a reference of its own."""
    for at in (5, 650, 651, 1290, 1546, 1547, 2303, 2314, 2319):
        one_far_key(kind, q_heads, 4, d, 2320, 5, [at] * 4, jump, 148)
