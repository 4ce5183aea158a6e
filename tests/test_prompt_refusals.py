"""Prompt attention and the store without a GPU: sizes, shapes and refusals of pools that have no device memory."""
import ctypes

import pytest

from paper_2512_09427_b200 import odma


def pool(dtype=odma.DTYPE_BF16, layers=2, kv_heads=4, head_dim=128, tokens=4096, **over):
    cfg = odma.config_default()
    cfg.safety_pct, cfg.max_len = 0, 2048
    for k, v in over.items():
        setattr(cfg, k, v)
    es = {odma.DTYPE_BF16: 2, odma.DTYPE_F32: 4, odma.DTYPE_FP8_E4M3: 1}[dtype]
    return odma.Pool(0, tokens * layers * 2 * kv_heads * head_dim * es, layers, kv_heads, head_dim, dtype, cfg)


def plan(p, new, ctx):
    for i, (a, c) in enumerate(zip(new, ctx)):
        assert p.alloc(i, a + c)[0] == odma.OK and (c == 0 or p.commit_step([i], [c]) == odma.OK)
    rc, t, _ = p.plan_host(list(range(len(new))), new)
    assert rc == odma.OK
    return t


def test_store_sizes():
    # the header's struct: two pointers, two 64-bit sizes, four 32-bit numbers
    assert ctypes.sizeof(odma.KvStore) == 48 and odma.KvStore.format.offset == 32 and odma.KvStore.n_layers.offset == 44
    p = pool()
    assert p.kv_store_bytes(odma.STORE_RAW, 0, 2, 10) == (2 * 2 * 10 * 4 * 256, 0)
    assert p.kv_store_bytes(odma.STORE_E4M3, 128, 1, 10) == (2 * 10 * 4 * 128, 2 * 10 * 4 * 4)
    assert p.kv_store_bytes(odma.STORE_INT8, 32, 2, 7) == (4 * 7 * 4 * 128, 4 * 7 * 4 * 16)
    assert p.kv_store_bytes(odma.STORE_INT4, 16, 2, 7) == (4 * 7 * 4 * 64, 4 * 7 * 4 * 32)
    assert p.kv_store_bytes(odma.STORE_INT4, 16, 1, 0) == (0, 0)
    assert pool(odma.DTYPE_FP8_E4M3, max_group=8).kv_store_bytes(odma.STORE_RAW, 0, 1, 3) == (2 * 3 * 4 * 128, 0)
    c, s = ctypes.c_uint64(), ctypes.c_uint64()
    for args in ((4, 32, 1, 1), (-1, 32, 1, 1), (1, 0, 1, 1), (1, 48, 1, 1), (1, 256, 1, 1), (1, 8, 1, 1), (1, 32, 0, 1), (1, 32, 3, 1), (1, 32, 1, -1),
                 (1, 32, 1, 1 << 40)):
        assert odma._lib.odma_kv_store_bytes(p._h, *args, ctypes.byref(c), ctypes.byref(s)) == odma.ERR_INVALID, args
    assert odma._lib.odma_kv_store_bytes(None, 0, 0, 1, 1, ctypes.byref(c), ctypes.byref(s)) == odma.ERR_INVALID
    assert odma._lib.odma_kv_store_bytes(p._h, 0, 0, 1, 1, None, ctypes.byref(s)) == odma.ERR_INVALID


def test_pools_without_memory_refuse_device_work():
    p = pool()
    t = plan(p, [5], [3])
    store = odma.KvStore(odma.STORE_RAW, 0, 0, 1, 256, 1 << 30)
    ids = (ctypes.c_uint64 * 1)(0)
    for f in (odma._lib.odma_pack_kv, odma._lib.odma_unpack_kv):
        assert f(p._h, ids, None, None, 1, ctypes.byref(store), None) == odma.ERR_INVALID
        assert f(None, ids, None, None, 1, ctypes.byref(store), None) == odma.ERR_INVALID
    assert odma._lib.odma_prefill_attention(p._h, 0, 256, 28, ctypes.byref(t), 256, 1 << 30, 512, None, None) == odma.ERR_INVALID
    assert odma._lib.odma_prefill_attention(None, 0, 256, 28, ctypes.byref(t), 256, 1 << 30, 512, None, None) == odma.ERR_INVALID


def test_workspace_sizes():
    p = pool()
    t = plan(p, [100, 1], [50, 900])
    full = p.prefill_workspace_bytes(28, t)
    # two partial results per share of a tile's rows (36 tokens of 7 heads), D + 2 floats each, and where the shares begin
    up = lambda b: (b + 255) // 256 * 256
    assert full == up(2 * 148 * 252 * 128 * 4) + up(2 * 148 * 252 * 8) + up(149 * 16)
    assert p.prefill_workspace_bytes(4, t) <= 2 * 148 * 256 * 130 * 4 + 2560 + 512
    for q_heads in (0, 3, 30, 4 * 9):
        assert p.prefill_workspace_bytes(q_heads, t) == 0
    assert odma._lib.odma_prefill_workspace_bytes(p._h, 28, None) == 0 and odma._lib.odma_prefill_workspace_bytes(None, 28, ctypes.byref(t)) == 0
    few = pool()
    assert few.prefill_workspace_bytes(28, plan(few, [1], [900])) < full // 20
    # an 8-bit pool: the batch's rows as bf16, of lengths rounded up to 16 at most
    q = pool(odma.DTYPE_FP8_E4M3, max_group=8)
    t8 = plan(q, [100, 1], [50, 900])
    rows = q.prefill_workspace_bytes(28, t8) - full
    assert 2 * 1051 * 4 * 128 * 2 <= rows <= 2 * (1051 + 30) * 4 * 128 * 2 + 256
    t8.reserved = 1                                  # a table of the device's: as many as the pool holds
    assert q.prefill_workspace_bytes(28, t8) - full == 2 * 4096 * 4 * 128 * 2
    t8.n = 5000
    assert q.prefill_workspace_bytes(28, t8) == 0
    for d in (16, 96, 256):
        o = pool(head_dim=d)
        assert o.prefill_workspace_bytes(4, plan(o, [2], [2])) == 0


@pytest.mark.parametrize("group,ok", [(1, True), (64, True), (65, False)])
def test_groups(group, ok):
    p = pool(kv_heads=1, max_group=80)
    assert (p.prefill_workspace_bytes(group, plan(p, [3], [3])) > 0) == ok
