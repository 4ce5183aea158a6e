"""Calls around slab attention next to one another: status words, streams, splits of a prefix and operands that overlap."""
import ctypes
import random

import pytest
import torch

import operator_refs as ref
from operator_refs import SlabPool

pytestmark = pytest.mark.gpu


def dev(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Refusal:
    """A device-built table one of whose requests is full, to set the status word with."""

    def __init__(self, s):
        self.s = s
        self.slabs, self.length = dev([[0, 16]]), dev([16])
        self.table = torch.empty(s.pool.tables_bytes(1), dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()

    def __call__(self, stream):
        self.s.pool.build_tables_device(self.slabs.data_ptr(), self.length.data_ptr(), 1, 1, self.table.data_ptr(), self.table.numel(),
                                        stream=stream)


# ---- the status word ---------------------------------------------------------------------------------

def test_status_is_taken_on_its_own_stream():
    """Read and cleared in the order of the given stream: work that other streams (the legacy one among them) still have to
    do is not waited for, and so cannot hold back the clearing either."""
    odma = ref.lib()
    s = SlabPool([64, 16], [40, 3], 1, 2, 64, "bf16")
    refuse, side = Refusal(s), torch.cuda.Stream()
    refuse(side.cuda_stream)
    assert s.pool.check_status(side.cuda_stream) == odma.ERR_OVERFLOW
    torch.cuda.synchronize()
    torch.cuda._sleep(1_000_000_000)                              # about half a second on the legacy stream
    done = torch.cuda.Event()
    done.record()
    refuse(side.cuda_stream)
    got = s.pool.check_status(side.cuda_stream), s.pool.check_status(side.cuda_stream)
    busy = not done.query()
    torch.cuda.synchronize()
    assert got == (odma.ERR_OVERFLOW, odma.OK) and busy


@pytest.mark.parametrize("kernel", ["mma", "tcgen05"])
def test_split_streams_right_behind_a_refusal(kernel):
    """The counts that split streams are merged by are nobody's but the decode launches'."""
    odma = ref.lib()
    lens = [3000, 5, 900]
    s = SlabPool([(x + 15) // 16 * 16 for x in lens], lens, 1, 2, 128, "bf16", ctas=24,
                 decode_kernel=odma.DECODE_TCGEN05 if kernel == "tcgen05" else odma.DECODE_MMA_SYNC)
    t = s.tables([0, 1, 2], [0, 0, 0])
    assert t.n_combine > 0
    q = s.randn(3, 14, 128)
    want, out = torch.empty_like(q), torch.empty_like(q)
    s.pool.decode_attention(0, q.data_ptr(), 14, t, want.data_ptr(), 0, s.stream)
    refuse, side = Refusal(s), torch.cuda.Stream().cuda_stream
    for i in range(60):
        out.fill_(float("nan"))
        torch.cuda.synchronize()
        refuse(side)
        assert s.pool.check_status(side) == odma.ERR_OVERFLOW
        s.pool.decode_attention(0, q.data_ptr(), 14, t, out.data_ptr(), 0, side)
        torch.cuda.synchronize()
        assert torch.equal(out, want), i
    assert s.pool.check_status(side) == odma.OK


@pytest.mark.parametrize("refused_first", [False, True])
def test_a_timeout_does_not_hide_a_refusal(refused_first):
    odma = ref.lib()
    s = SlabPool([64, 16], [40, 3], 1, 2, 64, "bf16")
    refuse = Refusal(s)
    if refused_first:
        refuse(s.stream)
    assert s.pool.selftest_timeout(5, s.stream) == odma.OK
    if not refused_first:
        refuse(s.stream)
    assert [s.pool.check_status(s.stream) for _ in range(3)] == [odma.ERR_TIMEOUT, odma.ERR_OVERFLOW, odma.OK]
