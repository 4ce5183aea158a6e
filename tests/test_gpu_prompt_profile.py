"""Launches of prompt attention and of the store are counted as their own."""
import pytest

from operator_refs import SlabPool, lib
from prompt_refs import Store, append_new, call_prefill, slab_rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind,ctas,new,launches", [("bf16", 148, [5, 3], 2), ("bf16", 2, [90, 300], 3), ("bf16", 1, [5, 3], 2), ("e4m3", 148, [5, 3], 3),
                                                    ("f32", 148, [5, 3], 2)])
def test_launches_are_counted(kind, ctas, new, launches):
    """Tiles and their merge; the counter's reset where tiles may be more than blocks; an 8-bit pool's widening; one block: no merge, and tiles may be more."""
    odma = lib()
    layers, launched = (3, 1) if kind == "e4m3" else (33, 2)         # of the store: 32 layers at a time
    s = SlabPool([128, 384], [20, 30], layers, 1, 64 if kind == "f32" else 128, kind, ctas=ctas)
    t = s.tables([0, 1], new)
    append_new(s, t, 0, new)
    q = s.randn(sum(new), 4, s.head_dim)
    counts = lambda: [s.pool.profile_read(k)[1] for k in (odma.K_DECODE, odma.K_COMBINE, odma.K_MIGRATE, odma.K_PREFILL, odma.K_STORE)]
    s.pool.profile_enable(True)
    call_prefill(s, 0, q, t)
    assert counts() == [0, 0, 0, launches, 0]
    store = Store(s, "raw", 0, 0, layers, 50)
    last = 2 * layers - 1
    before = slab_rows(s, last, 1, 0, 30)
    s.pool.pack_kv([0, 1], store.c, stream=s.stream)
    assert counts() == [0, 0, 0, launches, launched]
    s.pool.unpack_kv([1], Store(s, "raw", 0, 1, 1, 10).c, first=[5], count=[10], stream=s.stream)
    assert counts() == [0, 0, 0, launches, launched + 1]
    ms = s.pool.profile_read(odma.K_STORE)[0]
    assert 0 < ms < 1000 and s.pool.profile_read(odma.K_PREFILL)[0] > 0
    s.pool.profile_enable(False)
    assert s.sync() == 0 and (slab_rows(s, last, 1, 0, 30) == before).all()
