"""Host-side checks of cache weights and eviction: every call returns before anything reaches a device."""
import ctypes as C

import pytest

from tests.test_prefix_args import cache
from tests.test_relattn_args import FAKE, b, view  # noqa: F401


def weights(b, c=None, num_dst=3, dst_ptr=FAKE, heads=4, q=0, lse=FAKE, scale=0.125, decay=1.0, w=FAKE, out=FAKE, ws=FAKE, n=1 << 40):
    q = C.byref(view(b)) if q == 0 else C.byref(q) if q is not None else None
    p = C.c_void_p
    return b.load().tiga_mp_cache_weights(C.byref(c or cache(b)), num_dst, p(dst_ptr), heads, q, p(lse), scale, decay, p(w), p(out),
                                          p(ws), n, None)


def evict(b, c=None, w=FAKE, keep=10, recent=3, to=None, tw=FAKE, tl=FAKE, kept=FAKE, ws=FAKE, n=1 << 40):
    p = C.c_void_p
    return b.load().tiga_mp_cache_evict(C.byref(c or cache(b)), p(w), keep, recent, C.byref(to or cache(b, table=2 * FAKE)), p(tw), p(tl),
                                        p(kept), p(ws), n, None)


def test_weights(b):  # noqa: F811
    E, U, W = b.TIGA_EINVAL, b.TIGA_EUNSUPPORTED, b.TIGA_EWORKSPACE
    assert weights(b, c=cache(b, page_size=12)) == E and weights(b, c=cache(b, width=80)) == U and weights(b, heads=5) == E
    assert weights(b, num_dst=-1) == E and weights(b, num_dst=1 << 31) == U and weights(b, heads=0) == E
    assert weights(b, dst_ptr=None) == E and weights(b, c=cache(b, num_pages=0)) == E and weights(b, c=cache(b, length=None)) == E
    for s in (0.0, float("nan"), float("inf")):
        assert weights(b, scale=s) == E
    for s in (-0.5, float("nan"), float("inf")):
        assert weights(b, decay=s) == E and b"decay" in b.load().tiga_last_error()
    for bad in (None, view(b, data=FAKE + 8), view(b, row=12)):
        assert weights(b, q=bad) == E
    for bad in (0, FAKE + 4):
        assert weights(b, w=bad) == E and weights(b, out=bad) == E
    assert weights(b, lse=0) == E and weights(b, lse=FAKE + 2) == E
    assert weights(b, ws=0) == E and weights(b, ws=FAKE + 16) == E and weights(b, n=0) == W
    for over in (dict(batch=0), dict(kv_heads=0), dict(table_width=0)):
        heads = 0 if "kv_heads" in over else 4
        assert weights(b, c=cache(b, **over), heads=heads, q=None, lse=0, w=0, out=0, ws=0, n=0) == 0


def test_evict(b):  # noqa: F811
    E, U, W = b.TIGA_EINVAL, b.TIGA_EUNSUPPORTED, b.TIGA_EWORKSPACE
    assert evict(b, c=cache(b, page_size=12)) == E and evict(b, to=cache(b, page_size=12)) == E
    for over in (dict(batch=4), dict(kv_heads=4), dict(width=128), dict(dtype=1)):
        assert evict(b, to=cache(b, **over)) == E and b"differ" in b.load().tiga_last_error()
    assert evict(b, keep=0) == E and evict(b, keep=-1) == E and evict(b, recent=-1) == E and evict(b, recent=11) == E
    for side in ("c", "to"):
        for over in (dict(num_pages=0), dict(table=None), dict(k=view(b, data=FAKE + 8)), dict(v=view(b, row=0))):
            assert evict(b, **{side: cache(b, **over)}) == E, (side, over)
    assert evict(b, c=cache(b, length=None)) == E and evict(b, tl=0) == E and evict(b, tl=FAKE + 2) == E
    assert evict(b, w=0) == E and evict(b, w=FAKE + 4) == E and evict(b, tw=FAKE + 4) == E
    assert evict(b, kept=0) == E and evict(b, kept=FAKE + 1) == E
    assert evict(b, ws=0) == E and evict(b, ws=FAKE + 16) == E and evict(b, n=0) == W
    big = dict(batch=1 << 15, kv_heads=32)
    assert evict(b, c=cache(b, **big), to=cache(b, **big)) == U
    for over in (dict(batch=0), dict(kv_heads=0)):
        assert evict(b, c=cache(b, **over), to=cache(b, **over), w=0, tw=0, tl=0, kept=0, ws=0, n=0) == 0


def test_workspaces(b):  # noqa: F811
    L = b.load()
    size = lambda keep, to=None, **o: L.tiga_mp_cache_evict_workspace(C.byref(cache(b, **o)), C.byref(to or cache(b, **o)), keep)
    assert size(0) == 0 and size(10) >= 10 * 3 * 2 * (2 * 64 * 2 + 4)      # in place: the rows that stay
    assert all(size(k, batch=n) <= size(20, batch=3) for k in (1, 7, 20) for n in (1, 2, 3))
    other = cache(b, table=2 * FAKE)
    assert 0 < size(20, to=other) <= size(20)
    most = L.tiga_mp_cache_weights_workspace(C.byref(cache(b, batch=9, table_width=99)), 100, 32)
    for n in (0, 1, 40, 100):
        for batch in (1, 9):
            for h, hk in ((32, 2), (4, 4), (1, 1)):
                assert 0 < L.tiga_mp_cache_weights_workspace(C.byref(cache(b, batch=batch, table_width=9, kv_heads=hk)), n, h) <= most
