"""A workspace sized for a problem holds every smaller one: in any size, heads and source heads apart from each other."""
import ctypes as C
import itertools

import pytest

from tests.test_relattn_args import b, cache  # noqa: F401  (b: the fixture)

HEADS = [(1, 1), (2, 1), (2, 2), (12, 3), (12, 4), (12, 12), (16, 1), (16, 16), (32, 1), (32, 4), (32, 32)]


def pairs_hold(sizes):
    """sizes: {problem (a tuple of sizes): bytes}; every problem's bytes cover those of each smaller problem."""
    bad = [(small, big) for big, small in itertools.product(sizes, sizes)
           if all(x <= y for x, y in zip(small, big)) and sizes[small] > sizes[big]]
    assert not bad, f"{len(bad)} of {len(sizes)} squared, first: {bad[0]} {sizes[bad[0][0]]} > {sizes[bad[0][1]]}"
    assert min(sizes.values()) >= 256


@pytest.mark.parametrize("query", ["tiga_mp_attention_cross_fwd_workspace", "tiga_mp_attention_cross_bwd_workspace"])
def test_cross_attention(b, query):  # noqa: F811
    f = getattr(b.load(), query)
    pairs_hold({(n, s, batch, heads, kv, width): f(C.byref(b._Cross(n, s, batch, heads, kv, width, 0, None)))
                for n in (1, 5, 16, 17, 300) for s in (1, 64, 65, 129, 257, 1500) for batch in (1, 3, 70)
                for heads, kv in HEADS for width in (64, 128)})


def test_paged_attention(b):  # noqa: F811
    f = b.load().tiga_mp_attention_paged_fwd_workspace
    pairs_hold({(n, batch, table, heads, kv, width):
                f(C.byref(cache(b, batch=batch, table_width=table, kv_heads=kv, width=width)), n, heads)
                for n in (1, 2, 5, 16, 17, 300) for batch in (1, 3, 70) for table in (1, 5, 9, 17, 400)
                for heads, kv in HEADS for width in (64, 128)})


def test_fewer_source_heads_turn_narrow_tiles_wide(b):  # noqa: F811
    """The same heads over 32 and over 4 source heads: 16 and 128 rows to a source head."""
    L = b.load()
    cross = lambda kv: L.tiga_mp_attention_cross_fwd_workspace(C.byref(b._Cross(16, 1500, 1, 32, kv, 128, 0, None)))
    paged = lambda kv: L.tiga_mp_attention_paged_fwd_workspace(C.byref(cache(b, kv_heads=kv, width=128, table_width=400)), 16, 32)
    assert cross(32) >= cross(4) and paged(32) >= paged(4)
