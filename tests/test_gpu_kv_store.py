"""Rows of slabs to a store in fewer bits and back (odma_pack_kv, odma_unpack_kv) on the GPU, bit for bit."""
import ctypes
import math
import random

import pytest
import torch

from operator_refs import SlabPool, lib
from prompt_refs import Store, formats, quantised, restored, row_values, same_bits, slab_rows, up16

pytestmark = pytest.mark.gpu

FORMATS = [("raw", 16), ("e4m3", 16), ("e4m3", 128), ("int8", 32), ("int8", 128), ("int4", 16), ("int4", 32), ("int4", 64)]
POOLS = [("bf16", 4, 128), ("bf16", 3, 64), ("f32", 2, 64), ("f32", 1, 128), ("e4m3", 2, 128), ("bf16", 1, 48), ("f32", 5, 16), ("bf16", 2, 256)]


def check_pack(s, fmt, group, reqs, first, count, layer, n_layers, given=True):
    want_first = first or [0] * len(reqs)
    want_count = count or [s.lens[r] - f for r, f in zip(reqs, want_first)]
    st = Store(s, fmt, group, layer, n_layers, sum(want_count))
    before = s.mem.clone()
    s.pool.pack_kv(reqs, st.c, first, count, s.stream)
    assert s.sync() == 0
    assert torch.equal(s.mem.view(torch.uint8), before.view(torch.uint8))
    codes, scales = st.parts(s.kv_heads)
    for i, a in enumerate(st.arrays):
        rows = torch.cat([slab_rows(s, a, r, f, c) for r, f, c in zip(reqs, want_first, want_count)])
        if fmt == "raw":
            assert torch.equal(codes[i], rows.view(torch.uint8))
            continue
        c, sc = quantised(row_values(s, rows, a), fmt, group)
        assert same_bits(scales[i], sc), (a, (scales[i] - sc).abs().max())
        assert torch.equal(codes[i], c), a
    return st


def check_unpack(s, st, reqs, first, count):
    """Into slabs of `s` (any pool with the same heads): the rows named, and nothing else, become what the store holds."""
    want_first = first or [0] * len(reqs)
    host = s.mem.cpu().clone()
    codes, scales = st.parts(s.kv_heads)
    s.pool.unpack_kv(reqs, st.c, first, count, s.stream)
    assert s.sync() == 0
    for i, a in enumerate(st.arrays):
        x = codes[i].view(s.mem.dtype) if st.fmt == "raw" else s.stored(restored(codes[i], scales[i], st.fmt, st.group), a)
        if s.kind == "e4m3" and st.fmt != "raw":         # (not rounded to the io type on the way)
            inv = torch.ones(()) / torch.tensor((s.v_scale if a % 2 else s.k_scale)[a // 2], dtype=torch.float32)
            x = (restored(codes[i], scales[i], st.fmt, st.group) * inv).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
        at = 0
        for r, f, c in zip(reqs, want_first, count):
            for h in range(s.kv_heads):
                row = s.base[r] * s.kv_heads + h * s.caps[r] + f
                host[a, row:row + c] = x[at:at + c, h]
            at += c
    assert same_bits(s.mem.cpu(), host)


@pytest.mark.parametrize("kind,hkv,d,fmt,group", [p + f for p in POOLS for f in FORMATS if p[2] % f[1] == 0])
def test_pack_and_unpack(kind, hkv, d, fmt, group):
    lens = [1, 40, 16, 5, 0, 97]
    s = SlabPool([up16(x) + 16 for x in lens], lens, 3, hkv, d, kind, seed=group + hkv)
    st = check_pack(s, fmt, group, list(range(6)), None, None, 0, 3)
    # into another pool, other places
    caps = [128, 16, 64, 16, 16, 112]
    t = SlabPool(caps, [0] * 6, 3, hkv, d, kind)
    check_unpack(t, st, [1, 0, 2, 3, 4, 5], None, lens)
    # a part of some, of one layer, in another order
    st = check_pack(s, fmt, group, [5, 1, 5], [90, 0, 3], [7, 11, 64], 1, 1)
    check_unpack(t, st, [0, 5, 2], [100, 1, 0], [7, 11, 64])


@pytest.mark.parametrize("fmt,group", [("raw", 0), ("e4m3", 64), ("int4", 32)])
def test_many_requests_and_layers(fmt, group):
    r = random.Random(3)
    lens = [r.choice([0, 1, 2, 7, 16]) for _ in range(300)]
    s = SlabPool([16] * 300, lens, 35, 2, 64, "bf16")        # several launches along both
    st = check_pack(s, fmt, group, list(range(300)), None, None, 0, 35)
    t = SlabPool([16] * 300, [0] * 300, 35, 2, 64, "bf16")
    order = list(range(300))
    r.shuffle(order)
    check_unpack(t, st, order, None, lens)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["e4m3", "int8", "int4"])
def test_special_values(kind, fmt):
    s = SlabPool([32], [32], 1, 1, 64, kind)
    x = torch.randn(32, 64, generator=s.gen)
    x[0] = 0
    x[1, :32] = 0
    x[2, 3] = math.inf
    x[3, 40] = math.nan
    x[4] *= 2.0 ** -110                          # below the smallest group
    x[5] *= 2.0 ** -95
    x[6] = 1e38
    x[7, 0] = -3e38
    x[8] = torch.linspace(-1, 1, 64)
    x[9] = -0.0
    x[10, 32:] = 2.0 ** -100
    x[11] = 7.0 * torch.arange(64) / 64 - 3.5    # ties
    x[12] = torch.arange(64) - 31.5
    x[12, 0] = 127.0
    x[13] = -math.inf
    s.mem[0], s.mem[1] = x.to(s.io).cuda(), x.flip(0).to(s.io).cuda()
    st = check_pack(s, fmt, 32, [0], None, None, 0, 1)
    check_unpack(SlabPool([48], [0], 1, 1, 64, kind), st, [0], [10], [32])
    t = SlabPool([32], [0], 1, 1, 64, kind)
    check_unpack(t, st, [0], None, [32])
    got = t.mem[0].float().cpu()
    assert (got[0] == 0).all() and torch.isnan(got[2, :32]).all() and torch.isfinite(got[2, 32:]).all()
    assert torch.isnan(got[3, 32:]).all() and (got[4] == 0).all() and torch.isnan(got[13]).all()
    # a code is the nearest: off by half a step of the format at most, one rounding of the fp32 product and of the result
    ok = [i for i in range(32) if i not in (2, 3, 4, 10, 13)]
    a, b = x[ok].to(s.io).double(), got[ok].double()
    top = a.unflatten(-1, (2, 32)).abs().amax(-1, keepdim=True).expand(-1, -1, 32).flatten(1)
    step = {"int8": top / 254, "int4": top / 14, "e4m3": a.abs() * 2.0 ** -4 + top / 448 * 2.0 ** -10}[fmt]
    assert ((a - b).abs() <= step * (1 + 2.0 ** -20) + a.abs() * 2.0 ** -21 + b.abs() * torch.finfo(s.io).eps / 2).all()


@pytest.mark.parametrize("kind,hkv,d", [("bf16", 3, 64), ("f32", 1, 128), ("e4m3", 2, 128), ("bf16", 1, 48)])
@pytest.mark.parametrize("fmt", ["raw", "e4m3", "int8", "int4"])
def test_sixteen_bytes_of_alignment(kind, hkv, d, fmt):
    """Codes that begin 16 bytes behind a multiple of 32, scales 4 behind one of 16."""
    odma = lib()
    s = SlabPool([48, 32], [33, 21], 2, hkv, d, kind, seed=4)
    st = check_pack(s, fmt, 16, [0, 1], None, None, 0, 2)
    codes = torch.full((st.cb + 32,), 0xA5, dtype=torch.uint8, device="cuda")
    scales = torch.full((st.sb // 4 + 2,), -7.0, device="cuda")
    assert codes.data_ptr() % 32 == 0
    c = odma.KvStore(st.c.format, 16, 0, 2, codes.data_ptr() + 16, st.cb, scales.data_ptr() + 4, st.sb)
    s.pool.pack_kv([0, 1], c, stream=s.stream)
    t = [SlabPool([48, 32], [0, 0], 2, hkv, d, kind) for _ in range(2)]
    for pool, store in zip(t, (c, st.c)):
        pool.pool.unpack_kv([0, 1], store, count=[33, 21], stream=s.stream)
    assert s.sync() == 0
    assert torch.equal(codes[16:-16], st.codes[:st.cb]) and (codes[:16] == 0xA5).all() and (codes[-16:] == 0xA5).all()
    assert torch.equal(scales[1:-1], st.scales[:st.sb // 4]) and scales[0] == -7 and scales[-1] == -7
    assert torch.equal(t[0].mem.view(torch.uint8), t[1].mem.view(torch.uint8))


def test_captured_and_on_a_side_stream():
    s = SlabPool([64, 64], [33, 50], 2, 2, 64, "bf16")
    t = SlabPool([64, 64], [0, 0], 2, 2, 64, "bf16")
    st = Store(s, "int8", 64, 0, 2, 83)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        stream = torch.cuda.current_stream().cuda_stream
        s.pool.pack_kv([0, 1], st.c, stream=stream)
        t.pool.unpack_kv([1, 0], st.c, count=[33, 50], stream=stream)
    for i in range(3):
        for r in range(2):
            for h in range(2):
                at = s.base[r] * 2 + h * 64
                s.mem[:, at:at + s.lens[r]] = torch.randn(4, s.lens[r], 64, generator=s.gen).to(s.io).cuda()
        graph.replay()
        torch.cuda.synchronize()
        for a in range(4):
            for r in range(2):
                x = slab_rows(s, a, r, 0, s.lens[r])
                want = s.stored(restored(*quantised(x.float(), "int8", 64), "int8", 64), a)
                assert torch.equal(slab_rows(t, a, 1 - r, 0, s.lens[r]), want), (i, a, r)


def test_refusals():
    odma = lib()
    s = SlabPool([32, 48], [20, 40], 2, 2, 64, "bf16")
    st = Store(s, "int8", 32, 0, 2, 60)
    before = s.mem.clone()

    def rc(unpack=False, reqs=(0, 1), first=None, count=None, n=None, **kw):
        c = odma.KvStore(st.c.format, st.c.group, 0, 2, st.codes.data_ptr(), st.cb, st.scales.data_ptr(), st.sb)
        for k, v in kw.items():
            setattr(c, k, v)
        ids = (ctypes.c_uint64 * len(reqs))(*reqs)
        arr = lambda v: None if v is None else (ctypes.c_int32 * len(v))(*v)
        f = odma._lib.odma_unpack_kv if unpack else odma._lib.odma_pack_kv
        return f(s.pool._h, ids, arr(first), arr(count), len(reqs) if n is None else n, ctypes.byref(c), None)

    for kw in ({"format": 4}, {"format": -1}, {"group": 0}, {"group": 24}, {"group": 128}, {"group": 8}, {"layer": -1}, {"layer": 1}, {"n_layers": 0},
               {"n_layers": 3}, {"n_layers": 0x7FFFFFFF}, {"codes": None}, {"codes": st.codes.data_ptr() + 8}, {"codes_bytes": st.cb - 1},
               {"scales": None}, {"scales": st.scales.data_ptr() + 2}, {"scales_bytes": st.sb - 1}, {"n": 0}, {"n": -1},
               {"codes": s.mem.data_ptr()}, {"scales": s.mem.data_ptr() + 64}, {"codes": s.mem.data_ptr() - 16}, {"scales": st.codes.data_ptr() + 64},
               {"first": [-1, 0]}, {"count": [-1, 0]}, {"first": [21, 0]}):
        assert rc(**kw) == odma.ERR_INVALID, kw
        if "first" not in kw:
            assert rc(unpack=True, **{"count": [20, 40], **kw}) == odma.ERR_INVALID, kw
    assert rc(unpack=True, first=[-1, 0], count=[1, 1]) == odma.ERR_INVALID
    assert rc(reqs=(0, 7)) == odma.ERR_UNKNOWN_REQ and rc(unpack=True, reqs=(7, 0), count=[1, 1]) == odma.ERR_UNKNOWN_REQ
    # beyond what is committed, beyond the slab; the same token twice
    assert rc(count=[21, 1]) == odma.ERR_OVERFLOW and rc(first=[0, 40], count=[1, 1]) == odma.ERR_OVERFLOW
    assert rc(unpack=True, count=[33, 1]) == odma.ERR_OVERFLOW
    assert rc(first=[0x7FFFFFFF, 0], count=[1, 1]) == odma.ERR_OVERFLOW and rc(first=[0, 0], count=[0x7FFFFFFF, 1]) == odma.ERR_OVERFLOW
    assert rc(unpack=True, reqs=(0, 0), first=[0, 4], count=[5, 5]) == odma.ERR_INVALID
    torch.cuda.synchronize()
    assert torch.equal(s.mem.view(torch.int16), before.view(torch.int16)) and (st.codes == 0x7F).all() and torch.isnan(st.scales).all()
    # what may be asked for: nothing, the same request in two parts, a packed one several times
    assert rc(count=[0, 0], codes=None, scales=None) == odma.OK and rc(first=[20, 40]) == odma.OK
    assert rc(reqs=(0, 0, 1, 0), count=[20, 20, 0, 20]) == odma.OK
    assert rc(unpack=True, reqs=(0, 0), first=[10, 0], count=[10, 10]) == odma.OK
    assert s.sync() == 0
