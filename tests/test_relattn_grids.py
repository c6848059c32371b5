"""Backward passes of more tiles than one grid of threads counts are refused before anything reaches a device."""
import ctypes as C

import pytest

from tests.test_relattn_args import FAKE, b, view  # noqa: F401  (b: the fixture)


@pytest.mark.parametrize("over", [dict(num_dst=1 << 20, batch=1 << 11, num_src=5), dict(num_dst=1 << 20, batch=1 << 12, num_src=500),
                                  dict(num_dst=3, batch=1 << 12, num_src=1 << 20)])
@pytest.mark.parametrize("want", [(1, 0, 0), (0, 1, 1), (1, 1, 1)])
def test_backward(b, over, want):  # noqa: F811
    rel = b._Cross(**{**dict(heads=1, kv_heads=1, width=64, dtype=0, src_len=None), **over})
    v, p = C.byref(view(b)), C.c_void_p(FAKE)
    assert b.load().tiga_mp_attention_cross_bwd(C.byref(rel), v, v, v, v, p, v, 0.125, *(v if w else None for w in want), p,
                                                1 << 60, None) == b.TIGA_EUNSUPPORTED
    assert b"tiles" in b.load().tiga_last_error()
