"""The cache's description as the binding packs it is the structure of include/sara.h."""
import ctypes

import paper_2607_26253_gb300.operators as ops
import paper_2607_26253_gb300.sara as s


def test_packed_cache_is_the_structure():
    values = (1 << 40, 2 << 40, 3 << 40, 1 << 33, 5, 6, 7, 64, 1)
    packed = ops._pack_cache(*values)
    assert len(packed) == ctypes.sizeof(s.Kv8Cache)
    c = s.Kv8Cache.from_buffer_copy(packed)
    assert tuple(getattr(c, n) for n, _ in s.Kv8Cache._fields_) == values
