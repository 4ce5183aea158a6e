"""How many blocks of the plain-ALU prompt kernel a call counts on, by what its workspace holds."""
import pytest

from operator_refs import lib
from test_prompt_refusals import plan, pool


@pytest.mark.parametrize("kind,head_dim", [("f32", 32), ("f32", 64), ("f32", 128), ("bf16", 32)])
def test_a_share_for_every_block_that_an_sm_holds(kind, head_dim):
    """Registers allow two blocks of 256 threads, shared memory (228 KB, 1 KB of it for each block) as many as its rows
    leave room for: 64 rows of queries and of keys 4 elements apart, 64 of values, 64 x 64 weights."""
    odma = lib()
    p = pool(odma.DTYPE_F32 if kind == "f32" else odma.DTYPE_BF16, head_dim=head_dim)
    rows = 4 * (2 * 64 * (head_dim + 4) + 64 * head_dim + 64 * 68)
    blocks = min(2, 228 * 1024 // (rows + 1024))
    assert blocks == (1 if head_dim == 128 else 2)
    shares, part_rows = 148 * blocks, 64             # 16 tokens of 4 heads
    up = lambda b: (b + 255) // 256 * 256
    need = up((shares + 1) * 16 + 4) + up(2 * shares * part_rows * head_dim * 4) + up(2 * shares * part_rows * 8)
    assert p.prefill_workspace_bytes(16, plan(p, [100], [50])) == need
