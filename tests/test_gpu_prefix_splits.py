"""A shared prefix over few and many splits: forms of the tensor-core kernel that the number of shares, the length and the
workspace choose between, and merges of many parts."""
import pytest
import torch

from operator_refs import SlabPool
from test_gpu_operators import run_prefix

pytestmark = pytest.mark.gpu


def plan(q_heads, kv_heads, n, length, ctas):
    """(parts per row, steps in turn?) of the tensor-core form: the least of waves x a block's ns + parts x rows / 5."""
    tiles, rows = (length + 127) // 128, n * (q_heads // kv_heads)
    blocks, best = kv_heads * ((rows + 255) // 256), None
    for s in range(1, min(tiles, 128) + 1):
        waves, each = -(-blocks * s // ctas), -(-tiles // s)
        for turn in range(2 if rows <= 128 else 1):
            block = 7500 + 2 * each * 750 if turn else 6500 + 2 * each * (900 if rows <= 128 else 1100)
            parts = 2 * s if turn else s
            cost = waves * block + parts * n * q_heads // 5
            if best is None or cost < best[0]:
                best = cost, parts, turn
    return best[1:]


def widened(s, q_heads, n, length):
    """Bytes of the workspace before the parts, and of one part."""
    kv = 2 * s.kv_heads * ((length + 127) // 128 * 128) * s.head_dim * 2 if s.kind == "e4m3" else 0
    return kv, n * q_heads * (s.head_dim + 2) * 4


def growing(s, length, seed=3):
    """Keys of the prefix that turn along the sequence: scores of about half the rows rise step by step, the others fall."""
    g = torch.Generator().manual_seed(seed)
    for h in range(s.kv_heads):
        turn = torch.randint(0, 2, (s.head_dim,), generator=g) * 2.0 - 1.0
        x = 0.2 * torch.randn(length, s.head_dim, generator=g) + 5.0 * torch.arange(length)[:, None] / length * turn
        at = s.base[0] * s.kv_heads + h * s.caps[0]
        s.mem[0, at:at + length] = s.stored(x[:, None], 0)[:, 0].cuda()


def pool(kind, kv_heads, d, length, lens, ctas, seed=1):
    caps = [(length + 31) // 16 * 16] + [(x + 15) // 16 * 16 for x in lens]
    return SlabPool(caps, [length + 3] + lens, 1, kv_heads, d, kind, ctas=ctas, seed=seed)


# steps in turn on both lanes: few shares, few rows, long splits
IN_TURN = [("bf16", 28, 4, 128, 2, 1041, 8), ("e4m3", 28, 4, 128, 2, 1041, 8), ("bf16", 12, 2, 64, 2, 1041, 2), ("bf16", 4, 4, 128, 1, 600, 4),
           ("bf16", 16, 1, 64, 8, 1500, 2), ("bf16", 4, 4, 128, 2, 897, 4)]


@pytest.mark.parametrize("kind,q_heads,hkv,d,n,length,ctas", IN_TURN)
@pytest.mark.parametrize("qscale", [1.0, 40.0])
def test_steps_taken_in_turn(kind, q_heads, hkv, d, n, length, ctas, qscale):
    parts, turn = plan(q_heads, hkv, n, length, ctas)
    assert turn == 1 and parts % 2 == 0
    lens = [30 + 7 * i for i in range(n)]
    s = pool(kind, hkv, d, length, lens, ctas)
    head, part = widened(s, q_heads, n, length)
    assert s.pool.prefix_workspace_bytes(q_heads, n, length) == (head + parts * part + 255) // 256 * 256
    growing(s, length)
    # as planned; a workspace for an odd number of parts (one fewer is used); for one (no turns); lengths that end a lane early
    for space in (None, *[head + k * part for k in (3, 2, 1) if k <= parts]):
        run_prefix(s, list(range(1, n + 1)), lens, 0, length, q_heads, qscale=qscale, space=space, repeat=2)
    for shorter in (length - 64, length - 65, 513):
        run_prefix(s, list(range(1, n + 1)), lens, 0, shorter, q_heads, qscale=qscale)


@pytest.mark.parametrize("kind,d,q_heads,hkv,n,length,ctas", [("bf16", 64, 12, 2, 40, 1041, 2), ("bf16", 128, 28, 4, 40, 2000, 4),
                                                             ("e4m3", 128, 7, 1, 40, 2000, 2), ("bf16", 64, 16, 1, 12, 3001, 1),
                                                             ("bf16", 128, 16, 2, 33, 1100, 1)])
@pytest.mark.parametrize("qscale", [1.0, 40.0])
def test_two_row_tiles_over_long_splits(kind, d, q_heads, hkv, n, length, ctas, qscale):
    """More than 128 rows per KV head, tens of steps per block: every ring of stages wraps, references rise at every step."""
    assert plan(q_heads, hkv, n, length, ctas)[1] == 0 and n * q_heads // hkv > 128
    lens = [1 + (11 * i) % 50 for i in range(n)]
    s = pool(kind, hkv, d, length, lens, ctas)
    growing(s, length)
    run_prefix(s, list(range(1, n + 1)), lens, 0, length, q_heads, qscale=qscale, repeat=2)


@pytest.mark.parametrize("kind,q_heads,hkv,d,n,length,least", [("bf16", 16, 1, 128, 1, 5000, 33), ("bf16", 8, 1, 64, 8, 12000, 65),
                                                               ("e4m3", 8, 1, 128, 1, 16300, 65), ("f32", 4, 1, 64, 1, 5000, 33)])
def test_merges_of_many_parts(kind, q_heads, hkv, d, n, length, least):
    lens = [5 + i for i in range(n)]
    s = pool(kind, hkv, d, length, lens, 148)
    head, part = widened(s, q_heads, n, length)
    best = (s.pool.prefix_workspace_bytes(q_heads, n, length) - head) // part
    assert best >= least
    growing(s, length)
    for k in (best, 33, 32, 31, 9, 8):
        run_prefix(s, list(range(1, n + 1)), lens, 0, length, q_heads, qscale=4.0, space=head + k * part)
