"""Gradients of packed attention where finite operands have products past fp32's range (bfloat16 has its exponents): what a row
makes with keys that it does not see reaches nothing, and a row whose scores are not finite nothing but what it sees."""
import pytest
import torch

from tests import relattn_ref as R
from tests.packed_ref import Packed, check, reference

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16
BIG = 2.0 ** 100


def gradients(lib, s):
    y, lse = lib.tiga_mp_attention_packed_fwd(s.q, s.k, s.v, s.ptr_t, want_lse=True)
    g = lib.tiga_mp_attention_packed_bwd(s.q, s.k, s.v, y, lse, s.dy, s.ptr_t)
    torch.cuda.synchronize()
    return dict(g, y=y, lse=lse)


# row and a later key of the second sequence that a tile of 128 keys may hold both of; heads, source heads, width
PLACES = [(0, 1), (3, 90), (130, 131), (140, 255), (129, 200), (290, 299)]
FORMS = [(1, 1, 64), (2, 1, 128), (6, 2, 64), (3, 3, 128)]


@pytest.mark.parametrize("row,key", PLACES)
@pytest.mark.parametrize("H,Hk,D", FORMS)
def test_a_cotangent_and_a_value_that_it_does_not_see(lib, row, key, H, Hk, D):
    """<dy_i, v_j> is past the range for that pair alone, so all results are finite and the definition's."""
    s = Packed([20, 300, 40], H, Hk, D, BF16, seed=31)
    i, j = s.ptr[1] + row, s.ptr[1] + key
    s.dy[:, :, 7] = 0
    s.v[:, :, 7] = 0
    s.dy[0, i, 7] = BIG
    s.v[0, j, 7] = BIG
    check(lib, s, f"{(row, key, H, Hk, D)}")


@pytest.mark.parametrize("row,key", [(0, 0), (90, 3), (130, 130), (255, 140), (200, 2), (299, 298)])
@pytest.mark.parametrize("H,Hk,D", FORMS)
def test_a_score_past_the_range(lib, row, key, H, Hk, D):
    """Row i has no finite lse: keys after it get the other rows' gradients, and the other rows theirs."""
    s = Packed([20, 300, 40], H, Hk, D, BF16, seed=32)
    i, j = s.ptr[1] + row, s.ptr[1] + key
    s.q[:, :, 7] = 0
    s.k[:, :, 7] = 0
    s.q[0, i, 7] = BIG
    out, bound = reference(s, D ** -0.5)      # without the key's large element: the others do not see a difference
    s.k[0, j, 7] = BIG
    got = gradients(lib, s)
    others = [r for r in range(s.N) if r != i]
    after = [r for r in range(s.N) if r < s.ptr[1] or r > i]
    # the element of dq that the large one is a factor of is not looked at
    rest = [e for e in range(D) if e != 7]
    for n in ("y", "lse"):
        R.assert_within(got[n][:, others], out[n][:, others], bound[n][:, others], n)
    R.assert_within(got["dq"][:, others][..., rest], out["dq"][:, others][..., rest], bound["dq"][:, others][..., rest], "dq")
    for n in ("dk", "dv"):
        R.assert_within(got[n][:, after], out[n][:, after], bound[n][:, after], n)


@pytest.mark.parametrize("row,key", PLACES)
@pytest.mark.parametrize("H,Hk,D", FORMS)
def test_a_query_and_a_key_that_it_does_not_see(lib, row, key, H, Hk, D):
    """Their score is past the range, and no pair's."""
    s = Packed([20, 300, 40], H, Hk, D, BF16, seed=33)
    i, j = s.ptr[1] + row, s.ptr[1] + key
    s.q[:, :, 7] = 0
    s.k[:, :, 7] = 0
    s.q[0, i, 7] = BIG
    s.k[0, j, 7] = BIG
    check(lib, s, f"{(row, key, H, Hk, D)}")
