"""The operators around slab attention on the GPU: device-built tables, norm + rotation + append, attention behind a
shared prefix, and a run of them together."""
import ctypes
import random

import pytest
import torch

import operator_refs as ref
from operator_refs import SlabPool, within

pytestmark = pytest.mark.gpu


def dev(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


# ---- tables ------------------------------------------------------------------------------------

class TableCase:
    """Slabs laid out in a shuffled order, lengths and new tokens; the call and its outputs, with canaries behind them."""

    def __init__(self, n, kv_heads, ctas, seed, mean=300, one=False):
        r = random.Random(seed)
        self.n, self.kv_heads, self.ctas, self.r = n, kv_heads, ctas, r
        self.length = [r.choice([0, 0, 1, 63, 64, int(mean * r.paretovariate(1.3) / 3)]) for _ in range(n)]
        self.new = [1] * n if one else [r.choice([0, 1, 1, 2, 17]) for _ in range(n)]
        self.cap = [(a + b + 15) // 16 * 16 + 16 * r.randint(0, 3) for a, b in zip(self.length, self.new)]
        order = list(range(n))
        r.shuffle(order)
        self.base, at = [0] * n, 0
        for i in order:
            self.base[i], at = at, at + self.cap[i]
        self.tokens, self.n_new = max(16, at), sum(self.new)
        odma = ref.lib()
        cfg = odma.config_default()
        cfg.safety_pct, cfg.window, cfg.max_batch, cfg.plan_ctas = 0, 16, n, ctas
        self.mem = torch.empty(self.tokens * kv_heads * 2 * 8, dtype=torch.bfloat16, device="cuda")
        self.pool = odma.Pool(self.mem.data_ptr(), self.mem.numel() * 2, 1, kv_heads, 8, odma.DTYPE_BF16, cfg)
        assert self.pool.get_stats()["total_tokens"] == self.tokens
        self.stream = torch.cuda.current_stream().cuda_stream

    def call(self, one=False, in_place=False):
        nbytes = self.pool.tables_bytes(self.n)
        slabs = dev([[a, b] for a, b in zip(self.base, self.cap)])
        length, new = dev(self.length), dev(self.new)
        table = torch.full((nbytes // 4 + 4,), -77, dtype=torch.int32, device="cuda")
        nxt = length if in_place else torch.full((self.n + 4,), -77, dtype=torch.int32, device="cuda")
        slots, pos = (torch.full((self.n_new + 4,), -77, dtype=torch.int32, device="cuda") for _ in range(2))
        t = self.pool.build_tables_device(slabs.data_ptr(), length.data_ptr(), self.n, self.n_new, table.data_ptr(), nbytes,
                                          0 if one else new.data_ptr(), nxt.data_ptr(), slots.data_ptr(), pos.data_ptr(), self.stream)
        torch.cuda.synchronize()
        assert t.words * 4 <= nbytes
        # nothing behind the outputs has changed
        assert (table[t.words:] == -77).all() and (slots[self.n_new:] == -77).all() and (pos[self.n_new:] == -77).all()
        assert in_place or (nxt[self.n:] == -77).all()
        assert (t.n, t.n_new_total, t.n_ctas, t.one_new_each) == (self.n, self.n_new, self.ctas, int(one))
        return table[:t.words].tolist(), nxt[:self.n].tolist(), slots[:self.n_new].tolist(), pos[:self.n_new].tolist()

    def check(self, status=None, **kw):
        want = ref.device_tables(self.base, self.cap, self.length, self.new, self.n_new, self.tokens, self.kv_heads, self.ctas)
        got = self.call(**kw)
        for name, a, b in zip(("table", "lengths", "slots", "positions"), got, want):
            assert a == b, (name, next(i for i in range(len(a)) if a[i] != b[i]) if len(a) == len(b) else (len(a), len(b)))
        odma = ref.lib()
        assert self.pool.check_status(self.stream) == (odma.OK if status is None else status)


@pytest.mark.parametrize("n,kv_heads,ctas", [(1, 1, 1), (1, 4, 148), (2, 1, 3), (5, 3, 148), (31, 8, 7), (64, 4, 148),
                                             (257, 2, 148), (513, 1, 300), (1024, 4, 148), (4096, 2, 1024)])
def test_device_tables_match_the_reference(n, kv_heads, ctas):
    for seed in range(2 if n < 1000 else 1):
        TableCase(n, kv_heads, ctas, seed + 10 * n).check()
    TableCase(n, kv_heads, ctas, 5 * n, mean=4000, one=True).check(one=True, in_place=True)


def test_device_tables_of_empty_requests():
    c = TableCase(6, 2, 148, 3)
    c.length, c.new, c.n_new = [0] * 6, [0] * 6, 0
    c.check()
    c.length[4] = 1
    c.cap[4] = max(16, c.cap[4])
    if c.base[4] + c.cap[4] <= c.tokens:
        c.check(in_place=True)


@pytest.mark.parametrize("which", ["base", "unaligned", "end", "length", "negative length", "negative new", "rows", "huge new"])
def test_device_tables_refuse_a_bad_request(which):
    odma = ref.lib()
    for i in (0, 17, 40):
        c = TableCase(41, 2, 16, 99)
        if which == "base":
            c.base[i] = -16
        elif which == "unaligned":
            c.base[i] += 8
        elif which == "end":
            c.cap[i] = c.tokens - c.base[i] + 16
        elif which == "length":
            c.length[i] = c.cap[i] + 1
        elif which == "negative length":
            c.length[i] = -1
        elif which == "negative new":
            c.new[i] = -1
        elif which == "rows":
            c.new[i] = 5
            c.length[i] = 0
            c.cap[i] = 16
            c.base[i] = 0
            c.n_new = sum(c.new) - 1           # the last rows are missing: whoever holds them is refused
            c.new[40] = max(1, c.new[40])
            c.n_new = sum(c.new) - 1
        elif which == "huge new":
            c.new[i] = 0x7FFFFFFF
        c.check(status=odma.ERR_OVERFLOW)


def test_device_tables_refusals_of_the_call():
    odma = ref.lib()
    c = TableCase(8, 2, 16, 1)
    L, t = odma._lib, odma.Tables()
    buf = torch.zeros(1 << 16, dtype=torch.int32, device="cuda")
    b, nbytes = buf.data_ptr(), c.pool.tables_bytes(8)
    good = [c.pool._h, b, b + 256, b + 512, 8, 8, b + 4096, nbytes, None, None, None, None, ctypes.byref(t)]

    def rc(**ch):
        a = list(good)
        for k, v in ch.items():
            a[int(k[1:])] = v
        return L.odma_build_tables_device(*a)

    for ch in ({"a1": None}, {"a2": None}, {"a6": None}, {"a12": None}, {"a4": 0}, {"a4": 9}, {"a5": -1}, {"a7": nbytes - 4},
               {"a6": b + 4100}, {"a1": b + 4}, {"a2": b + 2}, {"a3": b + 1}, {"a8": b + 2}, {"a9": b + 2}, {"a10": b + 3},
               {"a3": None, "a5": 7}):
        assert rc(**ch) == odma.ERR_INVALID, ch
    ids = (ctypes.c_uint64 * 1)(5)
    assert L.odma_slab_table(c.pool._h, ids, 1, b, b, None) == odma.ERR_UNKNOWN_REQ
    assert L.odma_slab_table(c.pool._h, ids, 9, b, b, None) == odma.ERR_INVALID
    assert L.odma_slab_table(c.pool._h, ids, 1, b + 4, b, None) == odma.ERR_INVALID
    assert c.pool.check_status() == odma.OK


def device_plan(s, reqs, new=None, n_new=None, advance=False):
    """Tables of `reqs` through the device path."""
    slabs, length = torch.empty(len(reqs), 2, dtype=torch.int32, device="cuda"), torch.empty(len(reqs), dtype=torch.int32, device="cuda")
    s.pool.slab_table(reqs, slabs.data_ptr(), length.data_ptr(), s.stream)
    d_new = dev(new) if new is not None else None
    t = s.pool.build_tables_device(slabs.data_ptr(), length.data_ptr(), len(reqs), n_new if n_new is not None else (sum(new) if new else len(reqs)),
                                   s.table.data_ptr(), s.table.numel(), d_new.data_ptr() if new is not None else 0, stream=s.stream)
    s.keep = (slabs, length, d_new)
    return t


KINDS = [("f32", 64, 2, "auto"), ("bf16", 128, 7, "auto"), ("bf16", 128, 7, "tcgen05"), ("bf16", 64, 12, "tcgen05"), ("e4m3", 128, 7, "auto")]


def decode_cfg(kernel):
    return {"decode_kernel": ref.lib().DECODE_TCGEN05} if kernel == "tcgen05" else {}


@pytest.mark.parametrize("kind,d,g,kernel", KINDS)
@pytest.mark.parametrize("lens", [[1], [0, 5, 0], [700, 64, 1, 65, 0, 333], [3000], [40] * 33])
def test_decode_attention_from_device_tables(kind, d, g, kernel, lens):
    caps = [(x + 31) // 16 * 16 for x in lens]
    s = SlabPool(caps, lens, 1, 2, d, kind, ctas=12, seed=len(lens), **decode_cfg(kernel))
    reqs = list(range(len(lens)))
    t = device_plan(s, reqs, [0] * len(lens))
    q = s.randn(len(lens), 2 * g, d)
    out = torch.full_like(q, 7.0)
    lse = torch.full((len(lens), 2 * g), 7.0, device="cuda")
    s.pool.decode_attention(0, q.data_ptr(), 2 * g, t, out.data_ptr(), lse.data_ptr(), s.stream)
    assert s.sync() == 0
    want, wl, bound, lb = s.reference(0, q, reqs, lens)
    full = torch.tensor([x > 0 for x in lens])
    within(out[full.cuda()], want[full], bound[full], "out")
    within(lse[full.cuda()], wl[full], lb[full], "lse")
    # a request without a token has no item: its rows stay as they were
    assert (out[~full.cuda()] == 7.0).all() and (lse[~full.cuda()] == 7.0).all()


def test_append_kv_from_device_tables_skips_what_no_request_has():
    lens = [10, 0, 31, 7]
    s = SlabPool([32, 16, 32, 16], lens, 1, 2, 64, "bf16")
    before = s.mem.clone()
    new = [3, 2, 2, 0]                        # the third does not fit (31 + 2 > 32) and is refused
    t = device_plan(s, [0, 1, 2, 3], new, n_new=9)
    k, v = s.randn(9, 2, 64), s.randn(9, 2, 64)
    s.pool.append_kv(0, t, k.data_ptr(), v.data_ptr(), s.stream)
    assert s.sync() == ref.lib().ERR_OVERFLOW
    want = before.clone()
    for a, rows in ((0, k), (1, v)):
        for req, first, count in ((0, 0, 3), (1, 3, 2)):
            for h in range(2):
                at = s.base[req] * 2 + h * s.caps[req] + lens[req]
                want[a, at:at + count] = rows[first:first + count, h]
    assert torch.equal(s.mem.view(torch.int16), want.view(torch.int16))


# ---- norm, rotation, append ---------------------------------------------------------------------

def run_append(s, t, owner, position, q_heads, rot_dim, interleaved=False, section=(), norm=True, positions=None, fused=True,
               in_place=False, layer=0, eps=1e-6, scale=2.0):
    """Runs append_qkv on random rows and checks queries, slab rows and everything that must not change.
    owner, position per row (owner -1: no request)."""
    tokens, hkv, d = len(owner), s.kv_heads, s.head_dim
    odma = s.odma
    if fused:
        both = s.randn(tokens, q_heads + 2 * hkv, d, scale=scale)
        q, k, v = both[:, :q_heads], both[:, q_heads:q_heads + hkv], both[:, q_heads + hkv:]
        stride = (q_heads + 2 * hkv) * d
    else:
        q, k, v = s.randn(tokens, q_heads, d, scale=scale), s.randn(tokens, hkv, d, scale=scale), s.randn(tokens, hkv, d)
        stride = 0
    q0 = q.cpu().clone()
    wq, wk = (1 + 0.3 * s.randn(d).float()).to(s.io), (1 + 0.3 * s.randn(d).float()).to(s.io)
    pairs = rot_dim // 2
    freq = torch.tensor([1e6 ** (-2.0 * i / max(1, rot_dim)) for i in range(pairs)] or [0.0], dtype=torch.float32)
    axes = max(1, len(section))
    axis = torch.cat([torch.full((c,), a) for a, c in enumerate(section or [pairs])]).long()
    given = positions is not None
    pos = positions if given else torch.tensor(position).clamp(min=0)[None].expand(axes, tokens)
    d_pos, d_freq = pos.to(torch.int32).contiguous().cuda(), freq.cuda()
    q_out = q if in_place else torch.full((tokens, q_heads, d), 9.0, dtype=s.io, device="cuda")
    prep = odma.QkvPrep(rot_dim, interleaved, section, d_freq.data_ptr(), d_pos.data_ptr() if given else 0,
                        wq.data_ptr() if norm else 0, wk.data_ptr() if norm else 0, eps, stride, stride, stride)
    before = s.mem.clone()
    s.pool.append_qkv(layer, t, q.data_ptr(), k.data_ptr(), v.data_ptr(), q_out.data_ptr(), q_heads, prep, s.stream)
    torch.cuda.synchronize()
    live = torch.tensor([o >= 0 for o in owner])
    zq, sq = ref.prepared(q0, wq.cpu() if norm else None, eps, freq, pos, axis, rot_dim, interleaved)
    zk, sk = ref.prepared(k.cpu(), wk.cpu() if norm else None, eps, freq, pos, axis, rot_dim, interleaved)
    within(q_out[live.cuda()], zq[live], (ref.rounding(zq, s.io) + sq)[live], "queries")
    if not in_place:
        assert (q_out[~live.cuda()] == 9.0).all()
    after, touched = s.mem.cpu(), torch.zeros(s.mem.shape[:2], dtype=torch.bool)
    for a, z, slack in ((2 * layer, zk, sk), (2 * layer + 1, v.cpu().double(), torch.zeros_like(zk))):
        rows = torch.tensor([[s.base[o] * hkv + h * s.caps[o] + p for h in range(hkv)] for o, p in zip(owner, position) if o >= 0],
                            dtype=torch.long)
        if not rows.numel():
            continue
        touched[a, rows.flatten()] = True
        got, want, far = after[a][rows], z[live], slack[live]
        if s.kind == "e4m3":
            inv = (torch.ones(()) / torch.tensor((s.v_scale if a % 2 else s.k_scale)[layer])).double()
            want, far = (want * inv).clamp(-448, 448), far * inv + want.abs() * inv * 2.0 ** -24
            # half a step of a code: 2^-4 of the value, or half of the smallest step (2^-10)
            within(got.view(torch.float8_e4m3fn).float(), want, torch.maximum(want.abs() * 2.0 ** -4, torch.full_like(want, 2.0 ** -10)) + far, "codes")
        elif a % 2:
            assert torch.equal(got.double(), want)
        else:
            within(got, want, ref.rounding(want, s.io) + far, "keys")
    as_bytes = after.view(torch.uint8).view(*after.shape[:2], -1)
    assert torch.equal(as_bytes[~touched], before.cpu().view(torch.uint8).view(*after.shape[:2], -1)[~touched])
    return q_out


SHAPES = [("bf16", 28, 4, 128), ("bf16", 10, 2, 64), ("bf16", 3, 1, 32), ("bf16", 4, 4, 256), ("bf16", 2, 1, 80), ("bf16", 5, 5, 8),
          ("f32", 2, 1, 64), ("f32", 6, 2, 128), ("f32", 3, 3, 24), ("e4m3", 28, 4, 128), ("e4m3", 5, 1, 128)]


@pytest.mark.parametrize("kind,q_heads,hkv,d", SHAPES)
@pytest.mark.parametrize("interleaved", [False, True])
def test_append_qkv(kind, q_heads, hkv, d, interleaved):
    lens, new = [0, 17, 250, 5], [1, 30, 2, 16]
    s = SlabPool([64, 64, 256, 32], lens, 2, hkv, d, kind, seed=d)
    t = s.tables([0, 1, 2, 3], new)
    owner = [i for i, c in enumerate(new) for _ in range(c)]
    position = [lens[i] + j for i, c in enumerate(new) for j in range(c)]
    for rot, norm, fused, layer in ((d, True, True, 0), (0, True, False, 1), (d // 16 * 8, False, True, 1), (8, False, False, 0)):
        run_append(s, t, owner, position, q_heads, rot, interleaved, norm=norm, fused=fused, layer=layer)
    assert s.sync() == 0


@pytest.mark.parametrize("axes", [2, 3, 4])
def test_append_qkv_with_several_axes_and_far_positions(axes):
    lens, new = [3, 0], [40, 23]
    s = SlabPool([64, 32], lens, 1, 2, 128, "bf16", seed=axes)
    t = s.tables([0, 1], new)
    owner, position = [0] * 40 + [1] * 23, list(range(3, 43)) + list(range(23))
    g = torch.Generator().manual_seed(axes)
    pos = torch.randint(0, 1 << 20, (axes, 63), generator=g)
    pos[0, :5] = torch.tensor([0, 1, -7, (1 << 31) - 1, -(1 << 31)])
    section = [64 // axes] * (axes - 1)
    section += [64 - sum(section)]
    run_append(s, t, owner, position, 6, 128, False, section, positions=pos)
    run_append(s, t, owner, position, 6, 128, True, section[:-1] + [0] * (axes < 4) + section[-1:] if axes < 4 else section,
               positions=torch.cat((pos, pos[:1])) if axes < 4 else pos)


def test_append_qkv_decode_batch_with_device_tables():
    lens = [5, 0, 15, 16, 300, 31, 63, 1] * 5
    caps = [(x + 16) // 16 * 16 for x in lens]
    caps[3] = 16                                # full: this request is refused
    s = SlabPool(caps, lens, 1, 4, 128, "bf16")
    reqs = list(range(len(lens)))
    owner = reqs[:3] + [-1] + reqs[4:]
    run_append(s, device_plan(s, reqs), owner, lens, 28, 128)
    assert s.sync() == ref.lib().ERR_OVERFLOW


def test_append_qkv_ragged_device_tables_with_spare_rows():
    lens, new = [5, 0, 9, 100, 3], [0, 7, 0, 30, 0]
    s = SlabPool([16, 16, 16, 144, 16], lens, 1, 2, 64, "f32")
    run_append(s, device_plan(s, list(range(5)), new, n_new=41), [1] * 7 + [3] * 30 + [-1] * 4, list(range(7)) + list(range(100, 130)) + [0] * 4, 4, 64)
    assert s.sync() == 0


def test_append_qkv_many_requests_ragged():
    r = random.Random(8)
    new = [r.choice([0, 1, 2, 5]) for _ in range(1100)]
    lens = [r.randint(0 if c else 1, 20) for c in new]
    s = SlabPool([32] * 1100, lens, 1, 1, 32, "bf16")
    t = s.tables(list(range(1100)), new)
    run_append(s, t, [i for i, c in enumerate(new) for _ in range(c)], [lens[i] + j for i, c in enumerate(new) for j in range(c)], 2, 32)


def test_append_qkv_in_place_and_special_values():
    lens = [4, 9]
    s = SlabPool([16, 16], lens, 1, 2, 128, "bf16")
    t = s.tables([0, 1])
    run_append(s, t, [0, 1], lens, 8, 128, fused=False, in_place=True)
    # zeros through the norm stay zeros (eps keeps the root away from 0); an infinity stays in its own head
    q = torch.zeros(2, 8, 128, dtype=torch.bfloat16, device="cuda")
    q[1, 3, 5] = float("inf")
    k = torch.zeros(2, 2, 128, dtype=torch.bfloat16, device="cuda")
    w = torch.ones(128, dtype=torch.bfloat16, device="cuda")
    f = torch.ones(64, device="cuda")
    out = torch.empty_like(q)
    prep = s.odma.QkvPrep(128, False, (), f.data_ptr(), 0, w.data_ptr(), w.data_ptr())
    s.pool.append_qkv(0, t, q.data_ptr(), k.data_ptr(), k.data_ptr(), out.data_ptr(), 8, prep, s.stream)
    torch.cuda.synchronize()
    bad = torch.zeros(2, 8, dtype=torch.bool)
    bad[1, 3] = True
    assert not out.cpu()[~bad].any()
    assert s.sync() == 0


def test_append_qkv_refusals():
    s = SlabPool([32, 32], [4, 9], 1, 2, 64, "bf16", max_batch=2)
    t = s.tables([0, 1])
    odma, x = s.odma, torch.zeros(1 << 14, dtype=torch.bfloat16, device="cuda")
    b = x.data_ptr()
    before = s.mem.clone()

    def rc(layer=0, q=b, k=b, v=b, out=b + 8192, q_heads=4, tables=t, prep=None, **kw):
        p = prep or odma.QkvPrep(**{"rot_dim": 64, "inv_freq": b, **kw})
        return odma._lib.odma_append_qkv(s.pool._h, layer, ctypes.byref(tables), q, k, v, out, q_heads, ctypes.byref(p), None)

    for kw in ({"layer": 1}, {"layer": -1}, {"q": None}, {"k": None}, {"v": None}, {"out": None}, {"q": b + 8}, {"k": b + 2},
               {"v": b + 4}, {"out": b + 8}, {"q_heads": 3}, {"q_heads": 0}, {"rot_dim": 60}, {"rot_dim": 72}, {"rot_dim": -8},
               {"inv_freq": 0}, {"inv_freq": b + 2}, {"positions": b + 2}, {"q_norm": b + 8}, {"k_norm": b + 4},
               {"section": [16, 15]}, {"section": [40, -8]}, {"section": [16, 17]}, {"q_stride": 128}, {"k_stride": 120},
               {"q_stride": 260}, {"v_stride": 132}, {"pos_stride": 1}, {"q_norm": b, "eps": -1.0}, {"k_norm": b, "eps": float("nan")},
               {"q_norm": b, "eps": float("inf")}):
        assert rc(**kw) == odma.ERR_INVALID, kw
    for field, value in (("n_axes", 0), ("n_axes", 5), ("interleaved", 2)):
        p = odma.QkvPrep(rot_dim=64, inv_freq=b)
        setattr(p, field, value)
        assert rc(prep=p) == odma.ERR_INVALID, field
    p = odma.QkvPrep(rot_dim=64, inv_freq=b, section=[1 << 30, 1 << 30])
    p.section[0] = p.section[1] = 0x7FFFFFFF
    assert rc(prep=p) == odma.ERR_INVALID
    assert odma._lib.odma_append_qkv(s.pool._h, 0, ctypes.byref(t), b, b, b, b, 4, None, None) == odma.ERR_INVALID
    assert odma._lib.odma_append_qkv(s.pool._h, 0, None, b, b, b, b, 4, ctypes.byref(p), None) == odma.ERR_INVALID
    torch.cuda.synchronize()
    assert torch.equal(s.mem.view(torch.int16), before.view(torch.int16))
    wide = SlabPool([16], [3], 1, 1, 264, "bf16")                 # heads of more than 256 elements
    assert odma._lib.odma_append_qkv(wide.pool._h, 0, ctypes.byref(wide.tables([0])), b, b, b, b + 8192, 1,
                                     ctypes.byref(odma.QkvPrep()), None) == odma.ERR_INVALID


# ---- attention behind a shared prefix ---------------------------------------------------------------

def run_prefix(s, reqs, lens, prefix_req, prefix_len, q_heads, t=None, layer=0, qscale=1.0, space=None, want_lse=True, repeat=1):
    n = len(reqs)
    t = t or s.tables(reqs, [0] * n)
    q = s.randn(n, q_heads, s.head_dim, scale=qscale)
    nbytes = s.pool.prefix_workspace_bytes(q_heads, n, prefix_len) if space is None else space
    ws = torch.full((nbytes + 64,), 0xFF, dtype=torch.uint8, device="cuda")          # NaN, and a canary behind it
    res = []
    for _ in range(repeat):
        out, lse = torch.full_like(q, float("nan")), torch.full((n, q_heads), float("nan"), device="cuda")
        s.pool.decode_attention_prefix(layer, q.data_ptr(), q_heads, prefix_req, prefix_len, t, ws.data_ptr(), nbytes,
                                       out.data_ptr(), lse.data_ptr() if want_lse else 0, s.stream)
        res.append((out, lse))
    assert s.sync() == 0
    assert (ws[nbytes:] == 0xFF).all()
    for o, l in res[1:]:
        assert torch.equal(o, res[0][0]) and torch.equal(l, res[0][1])
    out, lse = res[0]
    want, wl, bound, lb = s.reference(layer, q, reqs, lens, prefix_req, prefix_len)
    within(out, want, bound, "out")
    if want_lse:
        within(lse, wl, lb, "lse")
    return out, lse


PREFIX_KINDS = [("bf16", 28, 4, 128), ("bf16", 4, 4, 128), ("bf16", 16, 1, 128), ("bf16", 12, 2, 64), ("bf16", 40, 2, 64),
                ("bf16", 6, 3, 32), ("f32", 2, 1, 64), ("f32", 6, 2, 128), ("f32", 3, 1, 32), ("e4m3", 28, 4, 128), ("e4m3", 3, 3, 128)]


@pytest.mark.parametrize("kind,q_heads,hkv,d", PREFIX_KINDS)
@pytest.mark.parametrize("prefix", [1, 15, 17, 64, 127, 128, 129, 300, 1041])
def test_attention_behind_a_prefix(kind, q_heads, hkv, d, prefix):
    lens = [1, 70, 16, 200, 33]
    s = SlabPool([(prefix + 31) // 16 * 16] + [(x + 15) // 16 * 16 for x in lens], [prefix + 3] + lens, 2, hkv, d, kind, seed=prefix, max_group=20)
    run_prefix(s, [1, 2, 3, 4, 5], lens, 0, prefix, q_heads, layer=1)


@pytest.mark.parametrize("kind,q_heads,hkv,d", [("bf16", 28, 4, 128), ("bf16", 12, 2, 64), ("f32", 2, 1, 64), ("e4m3", 28, 4, 128)])
@pytest.mark.parametrize("n", [1, 2, 19, 37, 75])
def test_attention_behind_a_prefix_batches(kind, q_heads, hkv, d, n):
    r = random.Random(n)
    lens = [r.randint(1, 90) for _ in range(n)]
    s = SlabPool([640] + [96] * n, [633] + lens, 1, hkv, d, kind, seed=n, ctas=20, max_batch=n)
    run_prefix(s, list(range(1, n + 1)), lens, 0, 633, q_heads, repeat=3)


@pytest.mark.parametrize("kind,d,kernel", [("f32", 64, "auto"), ("bf16", 128, "auto"), ("bf16", 128, "tcgen05"), ("e4m3", 128, "auto")])
def test_attention_behind_a_prefix_with_long_own_parts_and_empty_ones(kind, d, kernel):
    lens = [0, 1500, 0, 3, 700, 0]
    s = SlabPool([272] + [max(16, (x + 15) // 16 * 16) for x in lens], [260] + lens, 1, 2, d, kind, ctas=10, **decode_cfg(kernel))
    reqs = list(range(1, 7))
    run_prefix(s, reqs, lens, 0, 260, 6, device_plan(s, reqs, [0] * 6))
    # no prefix: the requests' own parts alone; zeros and -inf where there is nothing at all
    out, lse = run_prefix(s, reqs, lens, 0, 0, 6, device_plan(s, reqs, [0] * 6))
    assert not out[0].any() and (lse[0] == float("-inf")).all()


def test_a_prefix_of_the_slab_part_and_a_prefix_of_a_request_in_the_batch():
    s = SlabPool([512, 64, 64], [500, 40, 41], 1, 4, 128, "bf16")
    run_prefix(s, [1, 2], [40, 41], 0, 77, 28)
    run_prefix(s, [1, 2], [40, 41], 1, 40, 28, want_lse=False)


@pytest.mark.parametrize("kind,d", [("bf16", 128), ("bf16", 64), ("f32", 64), ("e4m3", 128)])
def test_attention_behind_a_prefix_large_scores(kind, d):
    # scores of some hundreds: the running maximum moves far from tile to tile, weights vanish
    lens = [30, 200]
    s = SlabPool([960, 48, 208], [950] + lens, 1, 2, d, kind, seed=4)
    run_prefix(s, [1, 2], lens, 0, 950, 8, qscale=40.0)


def test_prefix_workspace_smaller_and_refused():
    s = SlabPool([2048, 64, 64], [2000, 40, 41], 1, 4, 128, "bf16")
    one = 2 * 28 * (128 + 2) * 4
    best = s.pool.prefix_workspace_bytes(28, 2, 2000)
    assert best > 2 * one
    for space in (best, 2 * one, one + 8, one):
        run_prefix(s, [1, 2], [40, 41], 0, 2000, 28, space=space)
    odma, x = s.odma, torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    b, t = x.data_ptr(), s.tables([1, 2], [0, 0])

    def rc(layer=0, q=b, q_heads=28, req=0, length=2000, tables=t, ws=b, nbytes=best, out=b):
        return odma._lib.odma_decode_attention_prefix(s.pool._h, layer, q, q_heads, req, length, ctypes.byref(tables), ws, nbytes, out, None, None)

    for kw in ({"nbytes": one - 4}, {"nbytes": 0}, {"ws": None}, {"ws": b + 128}, {"layer": 1}, {"q": None}, {"q": b + 2}, {"out": None},
               {"q_heads": 27}, {"q_heads": 0}, {"length": -1}, {"tables": odma.Tables()}):
        assert rc(**kw) == odma.ERR_INVALID, kw
    assert rc(req=9) == odma.ERR_UNKNOWN_REQ
    assert rc(length=2001) == odma.ERR_OVERFLOW
    assert s.sync() == 0


# ---- together ---------------------------------------------------------------------------------------

@pytest.mark.parametrize("kind,q_heads,hkv,d", [("bf16", 28, 4, 128), ("f32", 2, 1, 64), ("e4m3", 28, 4, 128)])
def test_decode_loop_captured_once_and_replayed(kind, q_heads, hkv, d):
    """tables -> norm, rotation, append -> attention behind a prefix, as one graph whose replays advance the lengths."""
    lens = [0, 13, 64, 200]
    n, steps = len(lens), 4
    s = SlabPool([320] + [(x + steps + 15) // 16 * 16 for x in lens], [301] + lens, 1, hkv, d, kind, seed=2)
    odma, reqs = s.odma, [1, 2, 3, 4]
    slabs, length = torch.empty(n, 2, dtype=torch.int32, device="cuda"), torch.empty(n, dtype=torch.int32, device="cuda")
    s.pool.slab_table(reqs, slabs.data_ptr(), length.data_ptr(), s.stream)
    start = length.clone()
    pos = torch.empty(n, dtype=torch.int32, device="cuda")
    rows = torch.empty(n, q_heads + 2 * hkv, d, dtype=s.io, device="cuda")
    feed = [s.randn(n, q_heads + 2 * hkv, d) for _ in range(steps)]
    wq, wk = (1 + 0.1 * s.randn(d).float()).to(s.io), (1 + 0.1 * s.randn(d).float()).to(s.io)
    freq = torch.tensor([1e4 ** (-2.0 * i / d) for i in range(d // 2)], device="cuda")
    q = torch.empty(n, q_heads, d, dtype=s.io, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(n, q_heads, device="cuda")
    ws = torch.empty(s.pool.prefix_workspace_bytes(q_heads, n, 301), dtype=torch.uint8, device="cuda")
    stride = (q_heads + 2 * hkv) * d
    prep = odma.QkvPrep(d, False, (), freq.data_ptr(), pos.data_ptr(), wq.data_ptr(), wk.data_ptr(), 1e-6, stride, stride, stride)

    def step(stream):
        t = s.pool.build_tables_device(slabs.data_ptr(), length.data_ptr(), n, n, s.table.data_ptr(), s.table.numel(),
                                       d_len_next=length.data_ptr(), d_positions=pos.data_ptr(), stream=stream)
        es = rows.element_size()
        s.pool.append_qkv(0, t, rows.data_ptr(), rows.data_ptr() + q_heads * d * es, rows.data_ptr() + (q_heads + hkv) * d * es,
                          q.data_ptr(), q_heads, prep, stream)
        s.pool.decode_attention_prefix(0, q.data_ptr(), q_heads, 0, 301, t, ws.data_ptr(), ws.numel(), out.data_ptr(), lse.data_ptr(), stream)

    # eager
    results = []
    for i in range(steps):
        rows.copy_(feed[i])
        step(s.stream)
        torch.cuda.synchronize()
        results.append((q.clone(), out.clone(), lse.clone(), length.clone()))
    assert s.sync() == 0
    mem = s.mem.clone()
    now = [x + steps for x in lens]
    want, wl, bound, lb = s.reference(0, results[-1][0], reqs, now, 0, 301)
    within(results[-1][1], want, bound, "out")
    within(results[-1][2], wl, lb, "lse")
    # the last key rows are the prepared ones
    z, slack = ref.prepared(feed[-1][:, q_heads:q_heads + hkv].cpu(), wk.cpu(), 1e-6, freq.cpu(), torch.tensor(now)[None] - 1,
                            torch.zeros(d // 2, dtype=torch.long), d, False)
    if kind != "e4m3":
        for i, r in enumerate(reqs):
            got = torch.stack([s.values(0, r, h, now[i])[-1] for h in range(hkv)])
            within(got, z[i], ref.rounding(z[i], s.io) + slack[i], "key row")
    # captured, replayed over the same start
    length.copy_(start)
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        step(torch.cuda.current_stream().cuda_stream)
    for i in range(steps):
        rows.copy_(feed[i])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(length, results[i][3])
        for a, b in zip((q, out, lse), results[i]):
            assert torch.equal(a, b)
    assert torch.equal(s.mem.view(torch.uint8), mem.view(torch.uint8))
    # one step more than a slab holds: refused, flagged, and the others go on
    full = SlabPool([16, 16], [16, 3], 1, hkv, d, kind)
    t = device_plan(full, [0, 1])
    assert full.sync() == odma.ERR_OVERFLOW
    assert s.pool.commit_step(reqs, [steps] * n) == 0


def test_slab_table_is_not_captured():
    odma = ref.lib()
    s = SlabPool([64, 32], [40, 7], 1, 2, 64, "bf16")
    slabs, length = dev([[-1, -1], [-1, -1]]), dev([-1, -1])
    filled = torch.zeros(4, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        with pytest.raises(odma.OdmaError) as refusal:
            s.pool.slab_table([0, 1], slabs.data_ptr(), length.data_ptr(), torch.cuda.current_stream().cuda_stream)
        assert refusal.value.code == odma.ERR_INVALID
        filled.fill_(1.0)
    graph.replay()                                                # the capture has gone on
    torch.cuda.synchronize()
    assert filled.tolist() == [1.0] * 4 and length.tolist() == [-1, -1]
    for _ in range(8):                                            # and so do calls outside it, over every staging slot
        s.pool.slab_table([0, 1], slabs.data_ptr(), length.data_ptr(), s.stream)
    torch.cuda.synchronize()
    assert slabs.tolist() == [[0, 64], [64, 32]] and length.tolist() == [40, 7]


def test_on_another_stream():
    s = SlabPool([640, 64, 64], [633, 40, 41], 1, 4, 128, "bf16")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        s.stream = side.cuda_stream
        run_prefix(s, [1, 2], [40, 41], 0, 633, 28, device_plan(s, [1, 2], [0, 0]))
        s2 = SlabPool([64, 64], [40, 41], 1, 4, 128, "bf16")
        run_append(s2, device_plan(s2, [0, 1]), [0, 1], [40, 41], 28, 128)


# ---- large steps, and calls next to one another -------------------------------------------------------

MANY = [("bf16", 28, 4, 128, 128), ("bf16", 3, 1, 128, 16), ("bf16", 4, 2, 64, 8), ("bf16", 2, 1, 80, 80), ("bf16", 2, 1, 24, 8),
        ("bf16", 2, 2, 256, 128), ("f32", 4, 2, 64, 64), ("f32", 3, 3, 128, 24), ("e4m3", 8, 4, 128, 128), ("e4m3", 5, 1, 128, 40)]


@pytest.mark.parametrize("kind,q_heads,hkv,d,rot", MANY)
@pytest.mark.parametrize("interleaved", [False, True])
def test_append_qkv_of_a_large_chunk(kind, q_heads, hkv, d, rot, interleaved):
    lens, new = [0, 100, 7], [400, 1, 629]                        # 1,030 tokens: blocks of several, the last one short
    s = SlabPool([400, 112, 640], lens, 1, hkv, d, kind, seed=rot)
    t = s.tables([0, 1, 2], new)
    owner = [i for i, c in enumerate(new) for _ in range(c)]
    position = [lens[i] + j for i, c in enumerate(new) for j in range(c)]
    run_append(s, t, owner, position, q_heads, rot, interleaved, norm=rot % 16 == 0)
    pairs = rot // 2
    g = torch.Generator().manual_seed(d)
    run_append(s, t, owner, position, q_heads, rot, interleaved, [pairs - pairs // 2, pairs // 2], norm=rot % 16 != 0, fused=False,
               positions=torch.randint(0, 1 << 17, (2, 1030), generator=g))
    assert s.sync() == 0


def test_append_qkv_of_a_large_chunk_with_refused_and_spare_rows():
    lens, new = [5, 30, 0, 2], [300, 9, 500, 200]
    s = SlabPool([320, 32, 512, 208], lens, 1, 2, 128, "bf16")      # the second does not fit
    t = device_plan(s, [0, 1, 2, 3], new, n_new=1100)
    owner = [0] * 300 + [-1] * 9 + [2] * 500 + [3] * 200 + [-1] * 91
    position = list(range(5, 305)) + [0] * 9 + list(range(500)) + list(range(2, 202)) + [0] * 91
    run_append(s, t, owner, position, 4, 128)
    assert s.sync() == ref.lib().ERR_OVERFLOW


@pytest.mark.parametrize("kind,d,kernel", [("f32", 64, "auto"), ("bf16", 128, "auto"), ("bf16", 64, "mma"), ("bf16", 128, "mma"), ("e4m3", 128, "auto")])
def test_behind_a_prefix_nobody_holds_a_token(kind, d, kernel):
    over = {"decode_kernel": ref.lib().DECODE_MMA_SYNC} if kernel == "mma" else {}
    s = SlabPool([272, 16, 16, 16], [260, 0, 0, 0], 1, 2, d, kind, **over)
    run_prefix(s, [1, 2, 3], [0, 0, 0], 0, 260, 6, device_plan(s, [1, 2, 3], [0, 0, 0]))
    s = SlabPool([272, 64, 208, 16], [260, 50, 200, 1], 1, 2, d, kind, **over)
    run_prefix(s, [1, 2, 3], [50, 200, 1], 0, 260, 6, repeat=2)


@pytest.mark.parametrize("kind,d", [("bf16", 128), ("f32", 64), ("e4m3", 128)])
def test_a_prefill_chunk_behind_a_prefix(kind, d):
    """One stream per new token (the tables of a prefill chunk): token j sees the prefix, the request's tokens before the
    chunk and the chunk up to itself."""
    lens, new = [20, 0], [5, 9]
    s = SlabPool([144, 32, 16], [130, 25, 9], 1, 2, d, kind, max_batch=16)
    for r, have in ((1, 25), (2, 9)):                            # rows are there; lengths as before the chunk
        assert s.pool.free(r) == 0
        assert s.pool.set_buckets([s.caps[r]]) == 0
        rc, slab = s.pool.alloc(r, s.caps[r])
        assert rc == 0 and slab[0] == s.base[r]
    assert s.pool.commit_step([1], [20]) == 0
    t = s.pool.build_prefill_tables([1, 2], new, s.table.data_ptr(), s.table.numel(), s.stream)
    reqs = [1] * 5 + [2] * 9
    run_prefix(s, reqs, [lens[0] + j + 1 for j in range(5)] + [j + 1 for j in range(9)], 0, 130, 6, t)


@pytest.mark.parametrize("kind,q_heads,hkv,d", [("bf16", 28, 4, 128), ("bf16", 12, 2, 64), ("e4m3", 28, 4, 128)])
def test_steps_and_prefix_calls_in_a_row(kind, q_heads, hkv, d):
    """Decode steps (which may overlap with the launch before them) and calls behind a prefix, on two layers in turn,
    give the same bits whether or not every call is waited for."""
    lens = [30, 1, 400, 77, 130, 64]
    n, reqs = len(lens), [1, 2, 3, 4, 5, 6]

    def go(wait):
        s = SlabPool([320] + [(x + 47) // 16 * 16 for x in lens], [301] + lens, 2, hkv, d, kind, seed=9)
        ws = torch.empty(s.pool.prefix_workspace_bytes(q_heads, n, 301), dtype=torch.uint8, device="cuda")
        outs = []
        for i in range(6):
            for layer in (0, 1):
                q, k, v = s.randn(n, q_heads, d), s.randn(n, hkv, d), s.randn(n, hkv, d)
                a, b = torch.empty_like(q), torch.empty_like(q)
                t = s.pool.decode_step
                t(layer, 1, q_heads, reqs, q.data_ptr(), k.data_ptr(), v.data_ptr(), a.data_ptr(), 0, s.stream)
                if wait:
                    torch.cuda.synchronize()
                tab = s.tables(reqs)
                s.pool.decode_attention_prefix(1 - layer if i % 2 else layer, q.data_ptr(), q_heads, 0, 301, tab, ws.data_ptr(), ws.numel(),
                                               b.data_ptr(), 0, s.stream)
                if wait:
                    torch.cuda.synchronize()
                outs += [a, b, q, k, v]
            assert s.pool.commit_step(reqs, [1] * n) == 0
        assert s.sync() == 0
        return outs, s.mem.clone()

    # every layer's rows of a step are in place before the lengths move on: the calls on the other layer read rows of this step
    # that the step on that layer writes (i odd) or has written, so only equal schedules are compared
    one, mem1 = go(True)
    two, mem2 = go(True)
    for a, b in zip(one, two):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    three, mem3 = go(False)
    for a, b in zip(one, three):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    assert torch.equal(mem1.view(torch.uint8), mem3.view(torch.uint8))


def test_two_pools_on_two_streams():
    pools = [SlabPool([1040, 64, 240], [1033, 40, 230], 1, 4, 128, kind, seed=i) for i, kind in enumerate(("bf16", "e4m3"))]
    alone = [run_prefix(s, [1, 2], [40, 230], 0, 1033, 28) for s in pools]
    del alone
    qs = [s.randn(2, 28, 128) for s in pools]
    tabs = [s.tables([1, 2], [0, 0]) for s in pools]
    spaces = [torch.empty(s.pool.prefix_workspace_bytes(28, 2, 1033), dtype=torch.uint8, device="cuda") for s in pools]
    want = [torch.empty_like(q) for q in qs]
    for s, q, t, w, o in zip(pools, qs, tabs, spaces, want):
        s.pool.decode_attention_prefix(0, q.data_ptr(), 28, 0, 1033, t, w.data_ptr(), w.numel(), o.data_ptr(), 0, s.stream)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in pools]
    got = [[torch.empty_like(q) for _ in range(20)] for q in qs]
    for i in range(20):
        for s, q, t, w, o, st in zip(pools, qs, tabs, spaces, got, streams):
            s.pool.decode_attention_prefix(0, q.data_ptr(), 28, 0, 1033, t, w.data_ptr(), w.numel(), o[i].data_ptr(), 0, st.cuda_stream)
    torch.cuda.synchronize()
    for s, w, o in zip(pools, want, got):
        assert s.pool.check_status() == 0
        for x in o:
            assert torch.equal(x, w)
