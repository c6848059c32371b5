"""A row with lse = -inf gives no weight to any position, whatever its query holds."""
import pytest
import torch

from tests import relattn_ref as R
from tests.paged_ref import Batch
from tests.test_gpu_cache_weights import reference

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16

# lengths (with the new tokens, new tokens), heads, source heads, width, type; rows (sequence, token, head) that give nothing
CASES = [
    ([(300, 1), (40, 1)], 2, 1, 64, F16, [(0, 0, 1)]),
    ([(900, 3), (40, 2)], 4, 2, 128, BF16, [(0, 0, 0), (0, 2, 3), (1, 1, 1)]),
    ([(900, 300), (40, 1)], 2, 1, 64, BF16, [(0, 0, 0), (0, 100, 1), (0, 299, 0)]),
    ([(700, 257), (128, 128)], 8, 2, 128, F16, [(0, 5, 7), (0, 256, 0), (0, 256, 7), (1, 127, 3)]),
    ([(2000, 90), (60, 60)], 3, 1, 128, BF16, [(0, 0, 0), (0, 89, 2), (1, 0, 0), (1, 59, 1)]),
]


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("lens,H,Hk,D,dt,rows", CASES)
def test_rows_without_weight(lib, lens, H, Hk, D, dt, rows, bad):
    bt = Batch(lens, Hk, D, 16, dt, seed=61)
    q, cache = bt.tokens(H), bt.cache(lib)
    _, lse = lib.tiga_mp_attention_paged_fwd(cache, q, bt.dst_ptr, want_lse=True)
    for b, t, h in rows:
        lse[h, bt.ptr[b] + t] = float("-inf")
        q[h, bt.ptr[b] + t, 3:] = bad
    w = torch.rand(bt.num_pages, Hk, 16, generator=bt.g).cuda()
    got = lib.tiga_mp_cache_weights(cache, q, lse, bt.dst_ptr, w, torch.full_like(w, -7.0), 0.5)
    torch.cuda.synchronize()
    for b, t, h in rows:
        q[h, bt.ptr[b] + t] = 0      # for the oracle's sums of scores, which have no part in the result
    ref, bound = reference(bt, q, lse, w, 0.5, D ** -0.5)
    cells = ~torch.isnan(ref)
    R.assert_within(got.cpu()[cells], ref[cells], bound[cells], "weights")
