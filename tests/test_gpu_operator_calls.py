"""Calls around slab attention next to one another: status words, streams, splits of a prefix and operands that overlap."""
import ctypes

import pytest
import torch

import operator_refs as ref
from operator_refs import SlabPool
from test_gpu_operators import device_plan, run_prefix

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


# ---- append_qkv: where the queries may go ---------------------------------------------------------------

@pytest.mark.parametrize("kind,d", [("bf16", 64), ("f32", 32)])
def test_append_qkv_refuses_queries_over_rows_still_to_be_read(kind, d):
    """q_out is packed.  Over strided queries (or any other input) it lies on rows of tokens that other blocks still read."""
    s = SlabPool([32, 32, 32], [4, 9, 2], 1, 2, d, kind)
    odma, t = s.odma, s.tables([0, 1, 2])
    es, heads = s.mem.element_size(), 4
    row, kv, n = heads * d, 2 * d, 3
    x = torch.zeros(1 << 14, dtype=s.io, device="cuda")
    b = x.data_ptr() + 4096
    freq, pos = torch.ones(d // 2, device="cuda"), torch.zeros(64, dtype=torch.int32, device="cuda")
    far = x.data_ptr() + (x.numel() - n * row) * es              # behind everything else

    def rc(q, k, v, out, tables=t, **kw):
        p = odma.QkvPrep(**{"rot_dim": d, "inv_freq": freq.data_ptr(), **kw})
        return odma._lib.odma_append_qkv(s.pool._h, 0, ctypes.byref(tables), q, k, v, out, heads, ctypes.byref(p), s.stream)

    # one projection's output: [n, heads + 4 KV rows, d]
    wide = row + 2 * kv
    strides = {"q_stride": wide, "k_stride": wide, "v_stride": wide}
    fused = (b, b + row * es, b + (row + kv) * es)
    before = s.mem.clone()
    for out in (b, b + 16, b + row * es, b + (n - 1) * wide * es, b - (n * row - 8) * es, b + (n * wide - 8) * es):
        assert rc(*fused, out, **strides) == odma.ERR_INVALID, out - b
    # packed inputs
    packed = (b, b + n * row * es, b + n * (row + kv) * es)
    for out in (b + 16, b - 16, b + row * es, packed[1], packed[2], packed[2] + n * kv * es - 16):
        assert rc(*packed, out) == odma.ERR_INVALID, out - b
    for kw in ({"q_norm": far}, {"k_norm": far + (n * row - d) * es}, {"inv_freq": far + 16}, {"positions": far}):
        assert rc(*packed, far, **kw) == odma.ERR_INVALID, kw
    torch.cuda.synchronize()
    assert torch.equal(s.mem.view(torch.uint8), before.view(torch.uint8)) and not x.any()
    # side by side, in place, and in the gaps between strided rows
    assert rc(*fused, b - n * row * es, **strides) == odma.OK
    assert rc(*fused, b + n * wide * es, **strides) == odma.OK
    assert rc(*packed, b) == odma.OK
    assert rc(*packed, b - n * row * es) == odma.OK
    gap = wide + n * row
    assert rc(*fused, b + wide * es, q_stride=gap, k_stride=gap, v_stride=gap) == odma.OK
    one = SlabPool([32], [4], 1, 2, d, kind)
    p = odma.QkvPrep(rot_dim=d, inv_freq=freq.data_ptr(), positions=pos.data_ptr(), **strides)
    assert odma._lib.odma_append_qkv(one.pool._h, 0, ctypes.byref(one.tables([0])), *fused, b, heads, ctypes.byref(p), one.stream) == odma.OK
    assert s.sync() == 0 and one.sync() == 0

@pytest.mark.parametrize("which", ["q_stride", "k_stride", "v_stride", "pos_stride"])
def test_append_qkv_refuses_strides_beyond_any_memory(which):
    """Among them those whose bytes pass 64 bits."""
    s = SlabPool([32, 32], [4, 9], 1, 2, 64, "f32")
    odma, t = s.odma, s.tables([0, 1])
    x = torch.zeros(1 << 13, dtype=torch.float32, device="cuda")
    b = x.data_ptr()
    for stride in ((1 << 46) + 4, 1 << 60, 1 << 62, (1 << 63) - 4):
        p = odma.QkvPrep(rot_dim=64, inv_freq=b + 16384, positions=b + 20480, **{which: stride})
        assert odma._lib.odma_append_qkv(s.pool._h, 0, ctypes.byref(t), b, b + 4096, b + 8192, b + 24576, 4, ctypes.byref(p), s.stream) == odma.ERR_INVALID
    assert s.sync() == 0


# ---- tables ------------------------------------------------------------------------------------------

@pytest.mark.parametrize("new,after,cu,positions", [
    # five rows of four: counts as none, and request 3 has the last row
    ([3, 5, 0, 1, 0], [13, 0, 20, 8, 0], [0, 3, 3, 3, 4, 4], [10, 11, 12, 7]),
    # rows 3 and 4 of four: request 1 and whatever is behind it, with rows or without
    ([3, 2, 0, 1, 0], [13, 0, 0, 0, 0], [0, 3, 4, 4, 4, 4], [10, 11, 12, -1])])
def test_rows_that_do_not_fit_and_the_requests_behind_them(new, after, cu, positions):
    odma = ref.lib()
    lens = [10, 5, 20, 7, 0]
    s = SlabPool([32, 32, 32, 32, 16], lens, 1, 2, 64, "bf16")
    slabs = torch.empty(5, 2, dtype=torch.int32, device="cuda")
    length, nxt, slots, pos = torch.empty(5, dtype=torch.int32, device="cuda"), dev([-9] * 5), dev([-9] * 4), dev([-9] * 4)
    s.pool.slab_table(range(5), slabs.data_ptr(), length.data_ptr(), s.stream)
    d_new = dev(new)
    t = s.pool.build_tables_device(slabs.data_ptr(), length.data_ptr(), 5, 4, s.table.data_ptr(), s.table.numel(), d_new.data_ptr(),
                                   nxt.data_ptr(), slots.data_ptr(), pos.data_ptr(), s.stream)
    assert s.sync() == odma.ERR_OVERFLOW
    words = s.table.view(torch.int32).tolist()
    assert words[t.off_len:t.off_len + 5] == after and words[t.off_cu_new:t.off_cu_new + 6] == cu
    assert nxt.tolist() == [a or x for a, x in zip(after, lens)] and pos.tolist() == positions
    owner = [0, 0, 0, 3]
    assert slots.tolist() == [s.base[r] * 2 + p if p >= 0 else -1 for r, p in zip(owner, positions)]
    q = s.randn(5, 4, 64)
    out = torch.full_like(q, 7.0)
    s.pool.decode_attention(0, q.data_ptr(), 4, t, out.data_ptr(), 0, s.stream)
    assert s.sync() == odma.OK
    for r in (0, 2, 3):
        if after[r] == lens[r]:                                   # (rows of this step's tokens have not been written)
            want, _, bound, _ = s.reference(0, q[r:r + 1], [r], [lens[r]])
            ref.within(out[r:r + 1], want, bound, "out")
    assert (out[[r for r in range(5) if not after[r]]] == 7.0).all()


# ---- the late read-out on plans of the device ------------------------------------------------------------

@pytest.mark.parametrize("d,q_heads", [(128, 14), (64, 24)])
@pytest.mark.parametrize("lens", [[1], [0, 5, 0], [700, 64, 1, 65, 0, 333], [40] * 33])
def test_late_readout_from_device_tables_and_behind_a_prefix(d, q_heads, lens):
    """Shares without an item, many items per share, and every item left as a partial result."""
    odma = ref.lib()
    caps = [(x + 31) // 16 * 16 for x in lens] + [272]
    s = SlabPool(caps, lens + [260], 1, 2, d, "bf16", ctas=6, decode_kernel=odma.DECODE_TCGEN05, readout=odma.READOUT_LATE)
    n = len(lens)
    reqs = list(range(n))
    t = device_plan(s, reqs, [0] * n)
    q = s.randn(n, q_heads, d)
    out = torch.full_like(q, 7.0)
    s.pool.decode_attention(0, q.data_ptr(), q_heads, t, out.data_ptr(), 0, s.stream)
    assert s.sync() == odma.OK
    want, _, bound, _ = s.reference(0, q, reqs, lens)
    full = torch.tensor([x > 0 for x in lens])
    ref.within(out[full.cuda()], want[full], bound[full], "out")
    assert (out[~full.cuda()] == 7.0).all()
    run_prefix(s, reqs, lens, n, 260, q_heads, t, repeat=2)
