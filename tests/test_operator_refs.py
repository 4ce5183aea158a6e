"""The plain references of the operators checked against what defines them, and the operators' refusals on the host."""
import ctypes
import random

import pytest
import torch

import operator_refs as ref
from paper_2512_09427_b200 import odma


@pytest.mark.parametrize("ctas", [1, 3, 7, 148])
@pytest.mark.parametrize("n,kv_heads", [(1, 1), (2, 4), (9, 2), (60, 3)])
def test_device_table_reference_covers_every_token_once(n, kv_heads, ctas):
    r = random.Random(n * 1000 + kv_heads * 100 + ctas)
    length = [r.choice([0, 1, 63, 64, 65, r.randint(0, 2500)]) for _ in range(n)]
    new = [r.choice([0, 1, 1, 9]) for _ in range(n)]
    cap = [(a + b + 15) // 16 * 16 for a, b in zip(length, new)]
    base = [sum(cap[:i]) for i in range(n)]
    words, after, slots, pos = ref.device_tables(base, cap, length, new, sum(new), sum(cap), kv_heads, ctas)
    off_cta = 3 * ref.up4(n) + ref.up4(n + 1)
    off_items = off_cta + 12 * ctas
    off_comb = off_items + 8 * (n * kv_heads + ctas)
    items = [words[off_items + 8 * i:off_items + 8 * i + 8] for i in range(n * kv_heads + ctas)]
    live = [it for it in items if it[0] >= 0]
    assert [it[5] for it in sorted(live, key=lambda it: it[5])] == list(range(len(live)))
    seen = {}
    for it in sorted(live, key=lambda it: it[5]):
        seen.setdefault((it[0], it[1]), []).append(it)
        assert it[6] == base[it[0]] * kv_heads + it[1] * cap[it[0]] + it[2]
    for i in range(n):
        assert after[i] == length[i] + new[i]
        for h in range(kv_heads):
            run = seen.pop((i, h), [])
            assert sum(it[3] for it in run) == after[i]
            at = 0
            for it in run:
                assert it[2] == at and at % 64 == 0
                at += it[3]
            assert all((it[4] & 1) == (len(run) == 1) for it in run)
            assert [bool(it[4] & 2) for it in run] == [False] * (len(run) - 1) + [True] * bool(run)
            if len(run) > 1:
                assert min(it[3] for it in run[:-1]) >= 3 * 64
                rec = words[off_comb + 4 * run[0][7]:off_comb + 4 * run[0][7] + 4]
                assert rec == [i, h, run[0][5], len(run)] and len({it[7] for it in run}) == 1
                assert [it[5] for it in run] == list(range(rec[2], rec[2] + rec[3]))
            else:
                assert all(it[7] == -1 for it in run)
    assert not seen
    recs = [words[off_cta + 12 * c:off_cta + 12 * c + 12] for c in range(ctas)]
    assert recs[0][0] == 0 and recs[-1][1] == len(live) and all(a[1] == b[0] for a, b in zip(recs, recs[1:]))
    for r_ in recs:
        mine = items[r_[0]:r_[1]]
        assert r_[4:] == (mine[0] if mine else [0] * 8)
        split = [not it[4] & 1 for it in mine]
        assert split == sorted(split, reverse=True) and sum(split) <= 2
    assert sorted(p for p in pos) == sorted(length[i] + j for i in range(n) for j in range(new[i]))
    assert [s for s in slots] == [base[i] * kv_heads + length[i] + j for i in range(n) for j in range(new[i])]


def test_device_table_reference_refuses():
    ok = ([0, 32, 64], [32, 32, 32], [5, 6, 7], [1, 1, 1], 3, 96, 2, 4)
    assert ref.device_tables(*ok)[1] == [6, 7, 8]
    for which, i, value in ((0, 1, 40), (0, 1, -16), (1, 2, 48), (2, 1, 32), (2, 1, -1), (3, 1, -1), (3, 1, 4)):
        args = [list(a) if isinstance(a, list) else a for a in ok]
        args[which][i] = value
        words, after, slots, _ = ref.device_tables(*args)
        assert after[i] == args[2][i] and words[i] == words[4 + i] == words[8 + i] == 0
        assert after[0] == 6 and slots[0] == 5


def test_rotation_reference_is_a_rotation():
    g = torch.Generator().manual_seed(5)
    x = torch.randn(7, 3, 64, generator=g)
    f = torch.tensor([10.0 ** (-i / 4) for i in range(16)])
    pos = torch.randint(0, 1 << 20, (1, 7), generator=g)
    axis = torch.zeros(16, dtype=torch.long)
    for inter in (False, True):
        z, _ = ref.prepared(x, None, 0.0, f, pos, axis, 32, inter)
        assert torch.equal(z[..., 32:], x[..., 32:].double())
        assert torch.allclose(z.square().sum(-1), x.double().square().sum(-1), rtol=1e-12)
        back, _ = ref.prepared(z, None, 0.0, f, -pos, axis, 32, inter)
        assert torch.allclose(back, x.double(), atol=1e-12)
    # moving every position by the same amount leaves the products of queries and keys alone
    a, _ = ref.prepared(x, None, 0.0, f, pos, axis, 32, False)
    b, _ = ref.prepared(x, None, 0.0, f, pos + 977, axis, 32, False)
    assert torch.allclose(a[:, 0] @ a[:, 1].t(), b[:, 0] @ b[:, 1].t(), atol=1e-8)
    y, _ = ref.prepared(x, torch.ones(64), 0.0, f, pos, axis, 0, False)
    assert torch.allclose(y.square().mean(-1), torch.ones(7, 3, dtype=torch.float64))


def test_attention_reference_behind_a_prefix_is_attention_over_both():
    g = torch.Generator().manual_seed(6)
    q, k, v = (torch.randn(n, 32, generator=g) for n in (3, 50, 50))
    out, lse, _, _ = ref.attention(q, k, v, torch.float32)
    w = (q.double() @ k.double().t() / 32 ** 0.5)
    assert torch.allclose(out, torch.softmax(w, -1) @ v.double())
    assert torch.allclose(lse, w.exp().sum(-1).log())
    out, lse, _, _ = ref.attention(q, k[:0], v[:0], torch.float32)
    assert not out.any() and torch.isinf(lse).all()


def test_without_device_memory_the_operators_refuse():
    p = odma.Pool(0, 1 << 20, 1, 1, 64, odma.DTYPE_BF16)
    t, prep = odma.Tables(), odma.QkvPrep()
    L = odma._lib
    ids = (ctypes.c_uint64 * 1)(0)
    assert L.odma_slab_table(p._h, ids, 1, 256, 256, None) == odma.ERR_INVALID
    assert L.odma_build_tables_device(p._h, 256, 256, None, 1, 1, 256, 1 << 20, None, None, None, None, ctypes.byref(t)) == odma.ERR_INVALID
    assert L.odma_append_qkv(p._h, 0, ctypes.byref(t), 256, 256, 256, 256, 1, ctypes.byref(prep), None) == odma.ERR_INVALID
    assert L.odma_decode_attention_prefix(p._h, 0, 256, 1, 0, 0, ctypes.byref(t), 256, 256, 256, None, None) == odma.ERR_INVALID
    assert L.odma_prefix_workspace_bytes(None, 1, 1, 1) == 0


def test_prefix_workspace_sizes():
    cfg = odma.config_default()
    cfg.max_batch, cfg.max_group = 64, 8
    p = odma.Pool(0, 1 << 26, 1, 4, 128, odma.DTYPE_BF16, cfg)
    rows = 28 * 64 * (128 + 2) * 4
    assert p.prefix_workspace_bytes(28, 64, 1000) >= rows and p.prefix_workspace_bytes(28, 64, 1000) % 256 == 0
    assert p.prefix_workspace_bytes(28, 64, 0) == 256              # nothing to keep, and still a valid buffer
    # batches, lengths and head counts that the call refuses have no size
    for q_heads, n, length in ((27, 64, 10), (28, 65, 10), (28, 0, 10), (28, 64, -1), (28, 64, 1 << 30), (36, 1, 1), (0, 1, 1)):
        assert p.prefix_workspace_bytes(q_heads, n, length) == 0
    e = odma.Pool(0, 1 << 26, 1, 4, 128, odma.DTYPE_FP8_E4M3, cfg)
    assert e.prefix_workspace_bytes(28, 64, 1000) >= rows + 2 * 4 * 1024 * 128 * 2


def test_prep_structure_matches_the_header():
    assert ctypes.sizeof(odma.QkvPrep) == 8 * 8 + 8 * 4
    assert odma.QkvPrep(section=[16, 24, 24]).n_axes == 3 and odma.QkvPrep().n_axes == 1
