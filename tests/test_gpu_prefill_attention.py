"""Prompt attention over slabs (odma_prefill_attention) on the GPU against fp64."""
import ctypes
import random

import pytest
import torch

from operator_refs import SlabPool, within
from prompt_refs import append_new, call_prefill, prefill_reference, run_prefill, up16

pytestmark = pytest.mark.gpu

KINDS = [("bf16", 28, 4, 128), ("bf16", 4, 4, 128), ("bf16", 16, 1, 128), ("bf16", 12, 2, 64), ("bf16", 40, 2, 64), ("bf16", 64, 1, 64),
         ("bf16", 6, 3, 32), ("f32", 2, 1, 64), ("f32", 6, 2, 128), ("f32", 3, 1, 32), ("e4m3", 28, 4, 128), ("e4m3", 3, 3, 128)]


def pool_for(ctx, new, hkv, d, kind, **kw):
    return SlabPool([up16(a + b) + 16 * (i % 2) for i, (a, b) in enumerate(zip(ctx, new))], ctx, kw.pop("layers", 1), hkv, d, kind,
                    max_group=kw.pop("max_group", 64), **kw)


@pytest.mark.parametrize("kind,q_heads,hkv,d", KINDS)
@pytest.mark.parametrize("new", [1, 2, 17, 37, 130])
def test_prompts_of_one_request(kind, q_heads, hkv, d, new):
    for ctx in (0, 1, 127, 300):
        s = pool_for([ctx], [new], hkv, d, kind, seed=new + ctx, layers=2)
        run_prefill(s, [0], [ctx], [new], q_heads, layer=1, repeat=2)


@pytest.mark.parametrize("kind,q_heads,hkv,d", KINDS)
@pytest.mark.parametrize("ctas", [1, 3, 148])
def test_ragged_batches(kind, q_heads, hkv, d, ctas):
    r = random.Random(ctas)
    new = [0, 1, 64, 5, 129, 33, 0, 18, 1]
    ctx = [3, 0, 64, 700, 1, 129, 5, 0, 255]
    s = pool_for(ctx, new, hkv, d, kind, seed=r.randrange(1000), ctas=ctas)
    run_prefill(s, list(range(9)), ctx, new, q_heads)
