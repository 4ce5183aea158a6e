"""Prompt attention refuses results and workspaces that lie on what the call uses otherwise."""
import ctypes

import pytest
import torch

from operator_refs import SlabPool, lib, within
from prompt_refs import append_new, prefill_reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind,hkv,d", [("bf16", 2, 128), ("f32", 1, 64), ("e4m3", 2, 128)])
def test_overlaps_are_refused(kind, hkv, d):
    odma = lib()
    ctx, new, q_heads = [40, 9], [5, 70], 4
    s = SlabPool([48, 80], ctx, 1, hkv, d, kind, seed=2)
    t = s.tables([0, 1], new)
    append_new(s, t, 0, new)
    total, es = sum(new), torch.empty(0, dtype=s.io).element_size()
    need, rows = s.pool.prefill_workspace_bytes(q_heads, t), total * q_heads * d * es
    up = lambda n: (n + 255) // 256 * 256
    # one buffer, part by part: workspace, queries, results, log-sum-exps right behind one another
    at_q, at_out = need, need + rows
    at_lse, end = at_out + rows, at_out + rows + total * q_heads * 4
    buf = torch.zeros(up(end) + need, dtype=torch.uint8, device="cuda")
    q = s.randn(total, q_heads, d)
    buf[at_q:at_q + rows] = q.flatten().view(torch.uint8)
    b, pool, table, pool_bytes = buf.data_ptr(), s.mem.data_ptr(), s.table.data_ptr(), s.mem.numel() * s.mem.element_size()
    assert need % 256 == 0 and pool % 256 == 0 and table % 256 == 0

    def rc(space=b, out=b + at_out, lse=b + at_lse, queries=b + at_q):
        return odma._lib.odma_prefill_attention(s.pool._h, 0, queries, q_heads, ctypes.byref(t), space, need, out, lse, None)

    torch.cuda.synchronize()
    before, slabs = buf.clone(), s.mem.clone().view(torch.uint8)
    words = s.table.clone()
    bad = [{"space": at // 256 * 256} for at in (b + at_q, b + at_q + rows - 1, b + at_out, b + at_lse, b + end - 1)]
    bad += [{"space": pool}, {"space": (pool + pool_bytes - 1) // 256 * 256}, {"space": pool - 256}, {"space": table}, {"space": (table + 4 * t.words - 1) // 256 * 256}]
    bad += [{"lse": x} for x in (b, b + at_q - 4, b + at_q, b + at_out - 4, b + at_out, b + at_lse - 4, pool, pool + pool_bytes - 4, table, table + 4 * t.words - 4)]
    bad += [{"out": x} for x in (b, b + at_q, b + at_out - 16, b + at_out + 16, pool, pool + pool_bytes - 16, table, table + (4 * t.words - 1) // 16 * 16)]
    bad += [{"queries": x} for x in (b + need - 16, b + at_out + 16, b + at_out - 16)]
    for kw in bad:
        assert rc(**kw) == odma.ERR_INVALID, kw
    torch.cuda.synchronize()
    assert torch.equal(buf, before) and torch.equal(s.mem.view(torch.uint8), slabs) and torch.equal(s.table, words)
    assert rc() == odma.OK                           # side by side, nothing between them
    assert s.sync() == 0
    want = prefill_reference(s, 0, q, [0, 1], ctx, new)
    within(buf[at_out:at_lse].view(s.io).view(total, q_heads, d), want[0], want[2], "out")
    within(buf[at_lse:end].view(torch.float32).view(total, q_heads), want[1], want[3], "lse")
    assert torch.equal(buf[at_q:at_out], before[at_q:at_out])
    assert rc(lse=None) == odma.OK and rc(space=b + up(end)) == odma.OK and s.sync() == 0
