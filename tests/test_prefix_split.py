"""How a shared prefix is split where the plain ALUs compute it: as many blocks as an SM really holds."""
import pytest
import torch

import operator_refs as ref

SMS, ROWS = 148, 8
# blocks of 128 threads per SM by registers: 126 at head_dim 32, 150 and 156 (fp32) at 64 and 128
BLOCKS = {("f32", 32): 4, ("f32", 64): 3, ("f32", 128): 3, ("bf16", 32): 4}
SHAPES = [(2, 1, 4, 1000), (32, 8, 16, 1000), (32, 8, 64, 1000), (32, 8, 64, 4096), (8, 2, 64, 4096), (8, 2, 256, 2048), (16, 4, 4, 8192),
          (16, 4, 24, 2048), (5, 5, 1, 1), (5, 5, 3, 129)]


def pool_of(kind, head_dim, q_heads, kv_heads, n, length, device=False):
    odma = ref.lib()
    cfg = odma.config_default()
    cfg.safety_pct, cfg.window, cfg.max_batch, cfg.max_group, cfg.plan_ctas = 0, 16, n, q_heads // kv_heads, SMS
    es = 4 if kind == "f32" else 2
    nbytes = (length + 15) // 16 * 16 * 2 * kv_heads * head_dim * es
    mem = torch.empty(nbytes, dtype=torch.uint8, device="cuda") if device else None
    pool = odma.Pool(mem.data_ptr() if device else 0, nbytes, 1, kv_heads, head_dim, odma.DTYPE_F32 if kind == "f32" else odma.DTYPE_BF16, cfg)
    return pool, mem


def splits(kind, head_dim, q_heads, kv_heads, n, length):
    tiles, rows = (length + 127) // 128, n * (q_heads // kv_heads)
    blocks = kv_heads * ((rows + ROWS - 1) // ROWS)
    room = BLOCKS[kind, head_dim] * SMS

    def cost(s):
        return -(-blocks * s // room) * (3000 + 5000 * -(-tiles // s)) + s * n * q_heads // 5

    return min(range(1, min(tiles, 128) + 1), key=cost)


@pytest.mark.parametrize("kind,head_dim", sorted(BLOCKS))
@pytest.mark.parametrize("q_heads,kv_heads,n,length", SHAPES)
def test_splits_of_a_prefix_on_the_plain_alus(kind, head_dim, q_heads, kv_heads, n, length):
    pool, _ = pool_of(kind, head_dim, q_heads, kv_heads, n, length)
    part = n * q_heads * (head_dim + 2) * 4
    want = splits(kind, head_dim, q_heads, kv_heads, n, length) * part
    assert pool.prefix_workspace_bytes(q_heads, n, length) == max(256, (want + 255) // 256 * 256)


@pytest.mark.gpu
@pytest.mark.parametrize("kind,head_dim", sorted(BLOCKS))
def test_the_blocks_counted_on_are_the_ones_an_sm_holds(kind, head_dim):
    for q_heads, kv_heads, n, length in SHAPES:
        a, b = (pool_of(kind, head_dim, q_heads, kv_heads, n, length, device)[0] for device in (False, True))
        assert a.prefix_workspace_bytes(q_heads, n, length) == b.prefix_workspace_bytes(q_heads, n, length)
