"""Budgets that do not fit the C call's 32 bits are refused, not taken as what their low bits say."""
import pytest

from tests.test_relattn_args import b  # noqa: F401


@pytest.mark.parametrize("keep,recent", [((1 << 32) + 5, 0), (1 << 31, 0), (-(1 << 32) + 5, 0), (5, 1 << 32), (5, (1 << 32) + 3)])
def test_refused(b, keep, recent):  # noqa: F811
    with pytest.raises(ValueError, match="2\\^31"):
        b.tiga_mp_cache_evict(None, None, keep=keep, recent=recent)
