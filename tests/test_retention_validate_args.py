"""Host-side checks of the validation of a cache's pages: every call returns before anything reaches a device."""
import ctypes as C

from tests.test_prefix_args import cache
from tests.test_relattn_args import FAKE, b, view  # noqa: F401


def test_arguments(b):  # noqa: F811
    call = lambda **over: b.load().tiga_retention_validate(C.byref(cache(b, **over)), None)
    E, U = b.TIGA_EINVAL, b.TIGA_EUNSUPPORTED
    assert b.load().tiga_retention_validate(None, None) == E
    assert call(page_size=12) == E and call(width=80) == U and call(batch=1 << 16) == U and call(num_pages=0) == E
    assert call(table=None) == E and call(length=None) == E and call(length=FAKE + 2) == E and call(k=view(b, row=0)) == E
    assert call(batch=0, table=None) == 0 and call(kv_heads=0, length=None) == 0
