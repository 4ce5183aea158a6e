"""A request's way through the pool: its prompt in chunks, parked, back into another slab, on with the next chunk and the
decode, as a serving loop would call it; against fp64, and against the same without the parking."""
import pytest
import torch

from operator_refs import SlabPool, within
from prompt_refs import Store, append_new, call_prefill, prefill_reference, quantised, restored, slab_rows

pytestmark = pytest.mark.gpu


def chunk(s, reqs, ctx, new, q_heads, q, k, v):
    """One step of both layers: append, then attention of the chunk."""
    t = s.tables(reqs, new)
    outs = []
    for layer in range(2):
        s.pool.append_kv(layer, t, k[layer].data_ptr(), v[layer].data_ptr(), s.stream)
        out, lse = call_prefill(s, layer, q[layer], t)
        want = prefill_reference(s, layer, q[layer], reqs, ctx, new)
        within(out, want[0], want[2], f"out of layer {layer}")
        within(lse, want[1], want[3], f"lse of layer {layer}")
        outs.append(out)
    assert s.pool.commit_step(reqs, new) == 0
    return outs


@pytest.mark.parametrize("kind,q_heads,hkv,d", [("bf16", 28, 4, 128), ("f32", 4, 2, 64), ("e4m3", 8, 2, 128)])
@pytest.mark.parametrize("fmt,group", [("raw", 0), ("int8", 32), ("int4", 32)])
def test_prompt_parked_and_decoded(kind, q_heads, hkv, d, fmt, group):
    results = []
    for parked in (False, True):
        s = SlabPool([256, 128, 256], [0, 40, 0], 2, hkv, d, kind, seed=11, max_group=8)
        g = torch.Generator().manual_seed(5)
        rnd = lambda *shape: torch.randn(*shape, generator=g).to(s.io).cuda()
        first = chunk(s, [0, 1], [0, 40], [97, 20], q_heads, rnd(2, 117, q_heads, d), rnd(2, 117, hkv, d), rnd(2, 117, hkv, d))
        who = 0
        if parked:
            st = Store(s, fmt, group, 0, 2, 97)
            rows = [slab_rows(s, a, 0, 0, 97) for a in range(4)]
            s.pool.pack_kv([0], st.c, stream=s.stream)
            assert s.pool.free(0) == 0
            s.mem.view(torch.uint8)[:, s.base[0] * hkv:(s.base[0] + 256) * hkv] = 0x7F          # whoever has the slab next
            s.pool.unpack_kv([2], st.c, count=[97], stream=s.stream)
            assert s.pool.commit_step([2], [97]) == 0
            who = 2
            for a in range(4):
                if fmt == "raw":
                    assert torch.equal(slab_rows(s, a, 2, 0, 97), rows[a])
        second = chunk(s, [1, who], [60, 97], [3, 50], q_heads, rnd(2, 53, q_heads, d), rnd(2, 53, hkv, d), rnd(2, 53, hkv, d))
        # and a decode step of both
        t = s.tables([who, 1])
        q, k, v = rnd(2, q_heads, d), rnd(2, hkv, d), rnd(2, hkv, d)
        s.pool.append_kv(1, t, k.data_ptr(), v.data_ptr(), s.stream)
        out = torch.empty_like(q)
        s.pool.decode_attention(1, q.data_ptr(), q_heads, t, out.data_ptr(), 0, s.stream)
        assert s.sync() == 0
        want = s.reference(1, q, [who, 1], [148, 64])
        within(out, want[0], want[2], "decode")
        results.append(first + second + [out])
    if fmt == "raw":                                 # the rows are the same, and so is everything behind them
        for a, b in zip(*results):
            assert torch.equal(a, b)
