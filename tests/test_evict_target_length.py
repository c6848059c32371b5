"""The length array of the cache that rows are moved to is not read, so it need not be there; its other arrays need."""
import ctypes as C

from tests.test_prefix_args import cache
from tests.test_relattn_args import FAKE, b  # noqa: F401
from tests.test_retention_args import evict


def test_a_target_without_lengths(b):  # noqa: F811
    for length in (None, FAKE + 2):
        to = cache(b, table=2 * FAKE, length=length)
        assert evict(b, to=to, n=0) == b.TIGA_EWORKSPACE     # the last check before anything reaches a device
        assert evict(b, to=to, tl=0) == b.TIGA_EINVAL and evict(b, to=to, tl=FAKE + 2) == b.TIGA_EINVAL
        assert b.load().tiga_mp_cache_evict_workspace(C.byref(cache(b)), C.byref(to), 10) > 0
    assert evict(b, to=cache(b, table=None, length=None)) == b.TIGA_EINVAL
    assert evict(b, c=cache(b, length=None), to=cache(b, table=2 * FAKE)) == b.TIGA_EINVAL
