"""Prompt attention over slabs (odma_prefill_attention) on the GPU against fp64."""
import ctypes
import random

import pytest
import torch

from operator_refs import SlabPool, lib, within
from prompt_refs import append_new, call_prefill, causal, prefill_reference, run_prefill, up16

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


# ---- the split of the work ------------------------------------------------------------------------

@pytest.mark.parametrize("kind,q_heads,hkv,d", [("bf16", 28, 4, 128), ("bf16", 12, 2, 64), ("f32", 2, 1, 64), ("e4m3", 8, 1, 128)])
@pytest.mark.parametrize("ctas", [2, 31, 148, 300])
def test_few_tokens_behind_a_long_context(kind, q_heads, hkv, d, ctas):
    """Few rows, many keys: a tile is cut into many pieces."""
    for new, ctx in (([3], [2900]), ([1, 20], [1500, 2047]), ([40], [4200])):
        s = pool_for(ctx, new, hkv, d, kind, seed=ctx[0], ctas=ctas)
        run_prefill(s, list(range(len(new))), ctx, new, q_heads, repeat=3)


@pytest.mark.parametrize("kind,q_heads,hkv,d", [("bf16", 8, 2, 64), ("f32", 2, 2, 32), ("e4m3", 4, 2, 128)])
@pytest.mark.parametrize("n", [32, 33, 385, 1100])
def test_many_requests(kind, q_heads, hkv, d, n):
    """Up to 32 requests are planned by shuffles, more through scratch; some without new tokens, at the ends too."""
    r = random.Random(n)
    new = [r.choice([0, 0, 1, 1, 2, 9, 40]) for _ in range(n)]
    ctx = [r.choice([0, 1, 5, 130]) if a else r.randint(1, 9) for a in new]
    new[0] = new[-1] = 0
    ctx[0], ctx[-1] = 3, 7
    s = pool_for(ctx, new, hkv, d, kind, seed=n, max_batch=n)
    run_prefill(s, list(range(n)), ctx, new, q_heads)


@pytest.mark.parametrize("kind,q_heads,hkv,d", [("bf16", 28, 4, 128), ("bf16", 6, 6, 64), ("f32", 4, 2, 64)])
def test_one_long_prompt(kind, q_heads, hkv, d):
    new = 1283 if kind == "f32" else 2333
    s = pool_for([0], [new], hkv, d, kind, seed=5)
    run_prefill(s, [0], [0], [new], q_heads, repeat=2)


@pytest.mark.parametrize("kind,q_heads,hkv,d", [("bf16", 28, 4, 128), ("bf16", 12, 2, 64), ("e4m3", 8, 2, 128), ("f32", 4, 2, 64)])
@pytest.mark.parametrize("ctas", [2, 5, 148])
def test_more_tiles_than_blocks(kind, q_heads, hkv, d, ctas):
    """Blocks take tiles in an order that differs from run to run; short and long slabs, requests without new tokens."""
    r = random.Random(ctas)
    new = [300, 0, 1, 90, 700, 33, 250, 2, 0, 129] + [r.randint(1, 60) for _ in range(21)] + [400]
    ctx = [0, 4, 900, 513, 100, 0, 64, 0, 1, 250] + [r.choice([0, 40, 200]) for _ in range(21)] + [13]
    s = pool_for(ctx, new, hkv, d, kind, seed=ctas, ctas=ctas, max_batch=32)
    run_prefill(s, list(range(32)), ctx, new, q_heads, repeat=4)


@pytest.mark.parametrize("kind,q_heads,hkv,d", [("bf16", 28, 4, 128), ("e4m3", 28, 4, 128)])
@pytest.mark.parametrize("new,ctx", [([1500], [0]), ([1400], [4000]), ([2000, 18], [10, 3000]), ([1] * 30 + [1300, 0], [100] * 30 + [0, 7])])
def test_tiles_of_even_and_uneven_length(kind, q_heads, hkv, d, new, ctx):
    """Just more tiles than blocks: equal, rising, and one long one among short ones."""
    s = pool_for(ctx, new, hkv, d, kind, seed=new[0], max_batch=32)
    run_prefill(s, list(range(len(new))), ctx, new, q_heads, repeat=2)


# ---- scores that leave their reference ---------------------------------------------------------------

@pytest.mark.parametrize("kind,q_heads,hkv,d", [("bf16", 28, 4, 128), ("bf16", 12, 2, 64), ("f32", 2, 1, 64), ("e4m3", 8, 1, 128)])
@pytest.mark.parametrize("qscale,kscale", [(1.0, 9.0), (30.0, 1.0), (6.0, 6.0), (1e-3, 1e-3), (0.0, 1.0)])
def test_large_and_tiny_scores(kind, q_heads, hkv, d, qscale, kscale):
    new, ctx = [130, 33], [300, 129]
    s = pool_for(ctx, new, hkv, d, kind, seed=int(qscale), scale=kscale, ctas=40)
    run_prefill(s, [0, 1], ctx, new, q_heads, qscale=qscale, kscale=kscale, twice=True)


@pytest.mark.parametrize("kind,q_heads,hkv,d", [("bf16", 14, 2, 128), ("bf16", 8, 4, 64), ("f32", 4, 2, 64)])
@pytest.mark.parametrize("first,by", [(0, 32), (40, 32), (64, 64), (100, 3), (5, 128)])
def test_rising_scores(kind, q_heads, hkv, d, first, by):
    """Every `by` keys the scores rise by more than 16 powers of two: in a step's first and second half, and masked ones."""
    new, ctx = 150, 333
    s = pool_for([ctx], [new], hkv, d, kind, seed=by, ctas=7)
    t = s.tables([0], [new])
    append_new(s, t, 0, [new])
    u = torch.ones(d) / d ** 0.5
    n = ctx + new
    level = torch.clamp((torch.arange(n) - first).float().div(by).floor(), min=0) * 30.0          # of the scaled score
    level = torch.where(level > 1500, torch.full((), 1500.0), level)
    for h in range(hkv):
        at = h * s.caps[0]
        k = level[:, None] * u[None] * (d ** 0.5 / 4.0) + 0.1 * torch.randn(n, d, generator=s.gen)
        s.mem[0, at:at + n] = k.to(s.io).cuda()
    q = (u * 4.0 + 0.05 * torch.randn(new, q_heads, d, generator=s.gen)).to(s.io).cuda()
    got = call_prefill(s, 0, q, t)
    out, lse, bound, lse_bound = prefill_reference(s, 0, q, [0], [ctx], [new], twice=True)
    within(got[0], out, bound, "out")
    within(got[1], lse, lse_bound, "lse")


@pytest.mark.parametrize("kind,q_heads,hkv,d", [("bf16", 14, 2, 128), ("bf16", 4, 1, 64), ("f32", 4, 2, 64)])
def test_a_key_that_is_not_a_number(kind, q_heads, hkv, d):
    """It makes NaN of the tokens that see it, whichever unit takes its column, and of no other."""
    new, ctx = 200, 256
    for bad in list(range(128, 160)) + [3, 255, 256, 300, 455]:
        s = pool_for([ctx, 40], [new, 7], hkv, d, kind, seed=bad, ctas=5)
        t = s.tables([0, 1], [new, 7])
        append_new(s, t, 0, [new, 7])
        q = s.randn(new + 7, q_heads, d)
        clean = call_prefill(s, 0, q, t)
        s.mem[0, bad] = float("nan")                 # KV head 0
        out, lse = call_prefill(s, 0, q, t)
        g, hit = q_heads // hkv, max(0, bad - ctx)
        assert torch.isnan(out[hit:new, :g]).all() and torch.isnan(lse[hit:new, :g]).all(), bad
        assert torch.equal(out[:hit], clean[0][:hit]) and torch.equal(out[:, g:], clean[0][:, g:]) and torch.equal(out[new:], clean[0][new:])
        assert torch.equal(lse[:hit], clean[1][:hit])


def test_a_value_that_is_not_finite():
    """It reaches the tokens that see it, those of the same block of 128 keys in front of it, and no other request."""
    new, ctx = 300, 50
    s = pool_for([ctx, 40], [new, 64], 2, 128, "bf16", seed=3)
    t = s.tables([0, 1], [new, 64])
    append_new(s, t, 0, [new, 64])
    q = s.randn(new + 64, 8, 128)
    clean = call_prefill(s, 0, q, t)
    s.mem[1, 200] = float("inf")                     # KV head 0, position 200: of the block 128 .. 255
    out, lse = call_prefill(s, 0, q, t)
    assert not torch.isfinite(out[150:new, :4]).any()
    assert torch.equal(out[:128 - ctx], clean[0][:128 - ctx]) and torch.equal(out[:, 4:], clean[0][:, 4:]) and torch.equal(out[new:], clean[0][new:])
    assert torch.equal(lse, clean[1])


# ---- calls ---------------------------------------------------------------------------------------

def dev(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("kind,q_heads,hkv,d", [("bf16", 28, 4, 128), ("f32", 2, 1, 64), ("e4m3", 8, 2, 128)])
def test_device_tables_with_a_refused_request_and_spare_rows(kind, q_heads, hkv, d):
    """The refused request's rows of out and lse, and those that belong to none, stay as they were."""
    odma = lib()
    ctx, new = [20, 100, 0, 7], [33, 40, 5, 3]
    s = pool_for(ctx, new, hkv, d, kind, seed=9)
    slabs = [[s.base[i], s.caps[i]] for i in range(4)]
    slabs[1][1] = 128                                # 100 + 40 tokens do not fit
    total = sum(new) + 11
    table = torch.empty(s.pool.tables_bytes(4), dtype=torch.uint8, device="cuda")
    d_slabs, d_len, d_new = dev(slabs), dev(ctx), dev(new)
    t = s.pool.build_tables_device(d_slabs.data_ptr(), d_len.data_ptr(), 4, total, table.data_ptr(), table.numel(),
                                   d_n_new=d_new.data_ptr(), stream=s.stream)
    torch.cuda.synchronize()
    assert s.pool.check_status(s.stream) == odma.ERR_OVERFLOW
    k, v, q = s.randn(total, hkv, d), s.randn(total, hkv, d), s.randn(total, q_heads, d)
    s.pool.append_kv(0, t, k.data_ptr(), v.data_ptr(), s.stream)
    out, lse = call_prefill(s, 0, q, t, spare=11)
    assert (out[33:73] == -77).all() and (lse[33:73] == -77).all()
    keep = torch.cat((torch.arange(33), torch.arange(73, 81)))
    want = prefill_reference(s, 0, q[keep], [0, 2, 3], [20, 0, 7], [33, 5, 3])
    within(out[keep], want[0], want[2], "out")
    within(lse[keep], want[1], want[3], "lse")


@pytest.mark.parametrize("kind,q_heads,hkv,d", [("bf16", 28, 4, 128), ("e4m3", 28, 4, 128), ("f32", 4, 2, 64)])
def test_captured_steps(kind, q_heads, hkv, d):
    """Tables from device lengths, append and attention, captured once: each replay is the next chunk."""
    new, caps, steps = [19, 1, 64], [96, 48, 224], 3
    ctx = [5, 0, 30]
    s = SlabPool(caps, ctx, 1, hkv, d, kind, seed=2, max_group=64)
    total = sum(new)
    slabs, length, n_new = dev([[s.base[i], caps[i]] for i in range(3)]), dev(ctx), dev(new)
    table = torch.empty(s.pool.tables_bytes(3), dtype=torch.uint8, device="cuda")
    q, k, v = (torch.empty(total, h, d, dtype=s.io, device="cuda") for h in (q_heads, hkv, hkv))
    out, lse = torch.empty_like(q), torch.empty(total, q_heads, device="cuda")

    def step(stream, ws=None):
        t = s.pool.build_tables_device(slabs.data_ptr(), length.data_ptr(), 3, total, table.data_ptr(), table.numel(), n_new.data_ptr(),
                                       length.data_ptr(), stream=stream)
        if ws is None:
            return s.pool.prefill_workspace_bytes(q_heads, t)
        s.pool.append_kv(0, t, k.data_ptr(), v.data_ptr(), stream)
        s.pool.prefill_attention(0, q.data_ptr(), q_heads, t, ws.data_ptr(), ws.numel(), out.data_ptr(), lse.data_ptr(), stream)

    ws = torch.empty(step(s.stream), dtype=torch.uint8, device="cuda")
    length.copy_(dev(ctx))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(torch.cuda.current_stream().cuda_stream, ws)
    length.copy_(dev(ctx))
    for i in range(steps):
        for x in (q, k, v):
            x.copy_(s.randn(*x.shape))
        graph.replay()
        torch.cuda.synchronize()
        assert s.pool.check_status(s.stream) == 0
        before = [c + i * a for c, a in zip(ctx, new)]
        want = prefill_reference(s, 0, q, [0, 1, 2], before, new)
        within(out, want[0], want[2], f"out of replay {i}")
        within(lse, want[1], want[3], f"lse of replay {i}")
    assert length.tolist() == [c + steps * a for c, a in zip(ctx, new)]


def test_two_pools_on_two_streams():
    """Counts of cut tiles and workspaces are a pool's and a caller's own."""
    pools, want = [], []
    for i in range(2):
        s = pool_for([3000 + i], [50 + i], 4, 128, "bf16", seed=i)
        t = s.tables([0], [50 + i])
        append_new(s, t, 0, [50 + i])
        q = s.randn(50 + i, 28, 128)
        want.append(call_prefill(s, 0, q, t))
        ws = torch.empty(s.pool.prefill_workspace_bytes(28, t), dtype=torch.uint8, device="cuda")
        pools.append((s, t, q, ws, torch.empty_like(q), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(20):
        for s, t, q, ws, out, st in pools:
            s.pool.prefill_attention(0, q.data_ptr(), 28, t, ws.data_ptr(), ws.numel(), out.data_ptr(), 0, st.cuda_stream)
    torch.cuda.synchronize()
    for (s, _, _, _, out, _), (w, _) in zip(pools, want):
        assert torch.equal(out, w) and s.sync() == 0


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "f32"])
def test_a_request_named_several_times(kind):
    """Its slab is read for each; together they are longer than the pool."""
    s = pool_for([60], [20], 2, 128, kind, seed=1, max_batch=7)
    first = s.tables([0], [20])
    append_new(s, first, 0, [20])
    q = s.randn(20, 8, 128)
    want = call_prefill(s, 0, q, first)
    t = s.tables([0] * 7, [20] * 7)
    out, lse = call_prefill(s, 0, q.repeat(7, 1, 1), t)
    ref = prefill_reference(s, 0, q, [0], [60], [20])
    for i in range(7):                               # (cut at other places)
        within(out[20 * i:20 * i + 20], ref[0], ref[2], "out")
        within(lse[20 * i:20 * i + 20], ref[1], ref[3], "lse")
    within(want[0], ref[0], ref[2], "out")


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_two_calls_of_one_pool_at_once(kind):
    """Two layers on two streams, with a workspace each, as captured graphs too; what a workspace held before does not matter."""
    ctx, new = [100, 0, 7], [900, 400, 300]
    s = pool_for(ctx, new, 4, 128, kind, seed=6, layers=2)
    t = s.tables([0, 1, 2], new)
    calls = []
    for layer in range(2):
        append_new(s, t, layer, new)
        q = s.randn(sum(new), 28, 128)
        want = call_prefill(s, layer, q, t)
        ws = torch.full((s.pool.prefill_workspace_bytes(28, t),), 0xFF, dtype=torch.uint8, device="cuda")
        calls.append((layer, q, want, ws, torch.empty_like(q), torch.empty(sum(new), 28, device="cuda"), torch.cuda.Stream()))

    def run(c, stream):
        s.pool.prefill_attention(c[0], c[1].data_ptr(), 28, t, c[3].data_ptr(), c[3].numel(), c[4].data_ptr(), c[5].data_ptr(), stream)

    def check():
        torch.cuda.synchronize()
        for c in calls:
            assert torch.equal(c[4], c[2][0]) and torch.equal(c[5], c[2][1])
            c[4].zero_()
            c[3].fill_(0xFF)
        torch.cuda.synchronize()
        assert s.sync() == 0

    torch.cuda.synchronize()
    for _ in range(10):
        for c in calls:
            run(c, c[6].cuda_stream)
    check()
    graphs = []
    for c in calls:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            run(c, torch.cuda.current_stream().cuda_stream)
            run(c, torch.cuda.current_stream().cuda_stream)
    for _ in range(3):
        torch.cuda.synchronize()
        for c, g in zip(calls, graphs):
            with torch.cuda.stream(c[6]):
                g.replay()
                g.replay()
        check()


@pytest.mark.parametrize("kind,q_heads,hkv,d", [("bf16", 28, 4, 128), ("e4m3", 8, 2, 128), ("f32", 2, 1, 64)])
def test_single_tokens_agree_with_decode(kind, q_heads, hkv, d):
    ctx = [0, 1, 127, 128, 700, 2000]
    s = pool_for(ctx, [1] * 6, hkv, d, kind, seed=4)
    q, (out, _) = run_prefill(s, list(range(6)), ctx, [1] * 6, q_heads, want_lse=False)
    t = s.tables(list(range(6)), [1] * 6)
    other = torch.empty_like(out)
    s.pool.decode_attention(0, q.data_ptr(), q_heads, t, other.data_ptr(), 0, s.stream)
    assert s.sync() == 0
    want, _, bound, _ = prefill_reference(s, 0, q, list(range(6)), ctx, [1] * 6)
    within(other, want, bound, "decode")


@pytest.mark.parametrize("kind,q_heads,hkv,d", [("bf16", 28, 4, 128), ("bf16", 12, 2, 64), ("bf16", 6, 3, 32), ("f32", 2, 1, 64), ("e4m3", 8, 2, 128)])
def test_sixteen_bytes_of_alignment(kind, q_heads, hkv, d):
    """q and out begin 16 bytes behind a multiple of 32, lse 4 behind one of 16; whole tiles and cut ones."""
    for ctx, new in (([5, 0], [40, 300]), ([2500], [30])):
        s = pool_for(ctx, new, hkv, d, kind, seed=8)
        t = s.tables(list(range(len(new))), new)
        append_new(s, t, 0, new)
        total, shift = sum(new), 16 // torch.empty(0, dtype=s.io).element_size()
        q = s.randn(total * q_heads * d + shift, 1, 1).flatten()
        out = torch.full((total * q_heads * d + 2 * shift,), -7.0, dtype=s.io, device="cuda")
        lse = torch.full((total * q_heads + 2,), -7.0, device="cuda")
        ws = torch.empty(s.pool.prefill_workspace_bytes(q_heads, t), dtype=torch.uint8, device="cuda")
        assert q.data_ptr() % 32 == 0 and out.data_ptr() % 32 == 0
        s.pool.prefill_attention(0, q.data_ptr() + 16, q_heads, t, ws.data_ptr(), ws.numel(), out.data_ptr() + 16, lse.data_ptr() + 4, s.stream)
        assert s.sync() == 0
        want = call_prefill(s, 0, q[shift:].view(total, q_heads, d).clone(), t)
        assert torch.equal(out[shift:-shift], want[0].flatten()) and torch.equal(lse[1:-1], want[1].flatten())
        assert (out[:shift] == -7).all() and (out[-shift:] == -7).all() and lse[0] == -7 and lse[-1] == -7


def test_no_new_tokens_and_refusals():
    odma = lib()
    s = SlabPool([32, 32], [4, 9], 1, 2, 64, "bf16", max_batch=2, max_group=40)
    t = s.tables([0, 1], [3, 2])
    append_new(s, t, 0, [3, 2])
    x = torch.zeros(1 << 16, dtype=torch.bfloat16, device="cuda")
    b, out = x.data_ptr(), torch.full((5, 4, 64), -7.0, dtype=torch.bfloat16, device="cuda")
    need = s.pool.prefill_workspace_bytes(4, t)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")

    def rc(layer=0, q=b, q_heads=4, tables=t, space=ws.data_ptr(), nbytes=need, o=None, lse=None):
        return odma._lib.odma_prefill_attention(s.pool._h, layer, q, q_heads, ctypes.byref(tables) if tables else None, space, nbytes,
                                                out.data_ptr() if o is None else o, lse, None)

    for kw in ({"layer": 1}, {"layer": -1}, {"q": None}, {"q": b + 8}, {"o": out.data_ptr() + 4}, {"q_heads": 3}, {"q_heads": 0}, {"q_heads": 82},
               {"tables": None}, {"space": None}, {"space": ws.data_ptr() + 16}, {"nbytes": need - 1}, {"nbytes": 0}, {"lse": b + 2},
               {"o": b}, {"o": b + 5 * 4 * 64 * 2 - 16}, {"q": out.data_ptr() + 16}):
        assert rc(**kw) == odma.ERR_INVALID, kw
    torch.cuda.synchronize()
    assert (out == -7).all()
    assert rc(o=b + 5 * 4 * 64 * 2) == odma.OK and rc() == odma.OK
    none = s.tables([0, 1], [0, 0])
    out.fill_(-7)
    assert rc(tables=none, space=None, nbytes=0) == odma.OK
    torch.cuda.synchronize()
    assert (out == -7).all() and s.sync() == 0
    for d, group in ((96, 1), (64, 65)):             # head_dim, query heads per KV head
        o = SlabPool([16], [3], 1, 1, d, "bf16", max_group=80)
        to = o.tables([0], [1])
        assert o.pool.prefill_workspace_bytes(group, to) == 0
        assert odma._lib.odma_prefill_attention(o.pool._h, 0, b, group, ctypes.byref(to), ws.data_ptr(), need, out.data_ptr(), None, None) == odma.ERR_INVALID


def test_a_slab_beyond_32_bits():
    """Rows of the last array lie more than 2^32 elements behind the pool's first."""
    far, tail = 8_500_000, 4096
    odma = lib()
    cfg = odma.config_default()
    cfg.safety_pct, cfg.window, cfg.max_batch, cfg.max_len = 0, 16, 2, far
    T = far + tail
    mem = torch.empty(4, T, 128, dtype=torch.bfloat16, device="cuda")
    pool = odma.Pool(mem.data_ptr(), mem.numel() * 2, 2, 1, 128, odma.DTYPE_BF16, cfg)
    assert pool.set_buckets([tail, far // 16 * 16]) == 0
    assert pool.alloc(0, far // 16 * 16)[0] == 0
    rc, slab = pool.alloc(1, tail)
    assert rc == 0 and slab[0] == far // 16 * 16
    ctx, new, stream = 1000, 70, torch.cuda.current_stream().cuda_stream
    g = torch.Generator().manual_seed(1)
    rows = torch.randn(2, ctx + new, 128, generator=g).to(torch.bfloat16)
    mem[2:, slab[0]:slab[0] + ctx + new] = rows.cuda()
    assert pool.commit_step([1], [ctx]) == 0
    table = torch.empty(pool.tables_bytes(2), dtype=torch.uint8, device="cuda")
    t = pool.build_tables([1], table.data_ptr(), table.numel(), stream, [new])
    q = torch.randn(new, 4, 128, generator=g).to(torch.bfloat16).cuda()
    ws = torch.empty(pool.prefill_workspace_bytes(4, t), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)
    pool.prefill_attention(1, q.data_ptr(), 4, t, ws.data_ptr(), ws.numel(), out.data_ptr(), 0, stream)
    torch.cuda.synchronize()
    want, _, bound, _ = causal(q.cpu(), rows[0], rows[1], torch.bfloat16, torch.ones(ctx + new, dtype=torch.bool))
    within(out, want, bound, "out")
    # and the same rows to a store and back
    assert pool.commit_step([1], [new]) == 0
    n = 2 * (ctx + new) * 128 * 2
    codes = torch.zeros(n, dtype=torch.uint8, device="cuda")
    store = odma.KvStore(odma.STORE_RAW, 0, 1, 1, codes.data_ptr(), n)
    pool.pack_kv([1], store, stream=stream)
    mem[2:, slab[0]:slab[0] + ctx + new] = 0
    pool.unpack_kv([1], store, count=[ctx + new], stream=stream)
    torch.cuda.synchronize()
    assert torch.equal(codes.view(torch.bfloat16).view(2, ctx + new, 128).cpu(), rows)
    assert torch.equal(mem[2:, slab[0]:slab[0] + ctx + new].cpu(), rows)
