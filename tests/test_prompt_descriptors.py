"""Which descriptors prompt attention takes."""
import ctypes

import pytest

from operator_refs import lib
from test_prompt_refusals import plan, pool


def test_a_stream_per_token_has_no_workspace():
    odma = lib()
    p = pool()
    t = plan(p, [100, 1], [50, 900])
    assert t.reserved == 0 and p.prefill_workspace_bytes(28, t) > 0
    t.reserved = 2                                   # as odma_build_prefill_tables marks it
    assert p.prefill_workspace_bytes(28, t) == 0
    rc, none, _ = p.plan_host([0, 1], [0, 0])        # a step without new tokens is one all the same
    assert rc == odma.OK and none.reserved == 0 and none.n_new_total == 0 and p.prefill_workspace_bytes(28, none) > 0


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bf16", "f32", "e4m3"])
def test_a_stream_per_token_is_refused(kind):
    """odma_build_prefill_tables is for odma_decode_attention; the step's own descriptor is for odma_prefill_attention."""
    import torch
    from operator_refs import SlabPool, within
    from prompt_refs import append_new, call_prefill, prefill_reference

    odma = lib()
    s = SlabPool([64, 32], [4, 9], 1, 2, 128, kind, max_batch=16)
    other = torch.empty(s.pool.tables_bytes(2), dtype=torch.uint8, device="cuda")
    t = s.pool.build_tables([0, 1], other.data_ptr(), other.numel(), s.stream, [3, 2])
    append_new(s, t, 0, [3, 2])
    q = s.randn(5, 4, 128)
    per_token = s.pool.build_prefill_tables([0, 1], [3, 2], s.table.data_ptr(), s.table.numel(), s.stream)
    out = torch.full_like(q, -7.0)
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    for n_new_total in (0, 5):                       # as it is, and as a caller might try to mend it
        per_token.n_new_total = n_new_total
        assert odma._lib.odma_prefill_attention(s.pool._h, 0, q.data_ptr(), 4, ctypes.byref(per_token), ws.data_ptr(), ws.numel(), out.data_ptr(),
                                                None, None) == odma.ERR_INVALID
    per_token.n_new_total = 0
    torch.cuda.synchronize()
    assert (out == -7).all()
    s.pool.decode_attention(0, q.data_ptr(), 4, per_token, out.data_ptr(), 0, s.stream)
    got, _ = call_prefill(s, 0, q, t)
    assert s.sync() == 0
    want = prefill_reference(s, 0, q, [0, 1], [4, 9], [3, 2])
    within(out, want[0], want[2], "per token")
    within(got, want[0], want[2], "by tiles")
