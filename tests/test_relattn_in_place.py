"""Outputs in the place of inputs: taken where the strides agree, refused before anything reaches a device otherwise."""
import ctypes as C

import pytest

from tests.test_relattn_args import FAKE, b, cache, view  # noqa: F401  (b: the fixture)


@pytest.mark.parametrize("over", [dict(row=128), dict(head=1 << 10), dict(row=128, head=1 << 10)])
def test_paged_output_in_the_place_of_q(b, over):  # noqa: F811
    """y over q with other strides would write rows that other blocks have yet to read."""
    L, r, p = b.load(), C.byref, C.c_void_p(FAKE)

    def fwd(q, y, n=5, heads=4, nb=0):
        return L.tiga_mp_attention_paged_fwd(r(cache(b)), n, p, heads, r(q), 0.125, r(y), None, p, nb, None)

    q = view(b)
    assert fwd(q, view(b, **over)) == b.TIGA_EINVAL and b"in the place of q" in L.tiga_last_error()
    # a workspace of 0 bytes is the last thing that is refused: these get that far
    assert fwd(q, q) == b.TIGA_EWORKSPACE and fwd(q, view(b, data=2 * FAKE, **over)) == b.TIGA_EWORKSPACE
    assert fwd(q, view(b, batch=8)) == b.TIGA_EWORKSPACE                     # a packed axis has no batch stride
    # the stride of an axis with one entry is never used
    if "head" not in over:
        assert fwd(q, view(b, **over), n=1) == b.TIGA_EWORKSPACE
    if "row" not in over:
        assert fwd(q, view(b, **over), heads=2, n=5) == b.TIGA_EINVAL
