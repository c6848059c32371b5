"""Attention behind shared prefixes with lengths past the table, and with new tokens' pointers that overlap: more work than the host
knows of stays within the workspace, and the rows that see all of their positions are as ever."""
import pytest
import torch

from tests import relattn_ref as R
from tests.test_gpu_paged_attention import reference
from tests.test_gpu_prefix_attention import Grouped

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16
GUARD = 1 << 20

# positions of the table, sequences (new tokens), groups (sequences, shared), past: those whose length passes the table by how much,
# heads, source heads, width, page, type
CASES = [
    (256, [1], [(1, 50)], {0: 44}, 1, 1, 128, 16, F16),
    (4224, [1], [(1, 0)], {0: 776}, 32, 4, 128, 16, BF16),
    (512, [1, 1], [(2, 256)], {1: 1}, 3, 3, 64, 16, F16),
    (512, [1, 2, 1], [(3, 256)], {0: 900, 2: 5}, 5, 5, 64, 32, BF16),
    (1024, [1] * 7, [(3, 640), (2, 128)], {1: 1 << 20, 4: 3, 6: 1}, 6, 3, 128, 64, BF16),
    (2048, [40, 30], [(2, 1024)], {1: 70}, 4, 1, 128, 16, F16),
    (256, [1], [(1, 0)], {0: (1 << 31) - 300}, 2, 1, 64, 16, F16),
]


def make(positions, new, groups, past, Hk, D, page, dt):
    bt = Grouped([(positions - 7 * b, c) for b, c in enumerate(new)], groups, Hk, D, page, dt, seed=41)
    bt.table = bt.table[:, : positions // page].contiguous()
    for b, n in past.items():
        bt.length[b] = positions + n
    return bt


def guarded(lib, bt, q, H, fill):
    cache, C = bt.cache(lib), lib.C
    prefix = lib._prefix(cache, bt.group_ptr, bt.group_len)
    size = lib.load().tiga_mp_attention_prefix_fwd_workspace(cache.ref, C.byref(prefix), bt.num_dst, H)
    whole = torch.full((size + GUARD,), fill, dtype=torch.uint8, device="cuda")
    out = lib.tiga_mp_attention_prefix_fwd(cache, q, bt.dst_ptr, bt.group_ptr, bt.group_len, want_lse=True, ws=whole[:size])
    torch.cuda.synchronize()
    assert (whole[size:] == fill).all()
    return out


@pytest.mark.parametrize("positions,new,groups,past,H,Hk,D,page,dt", CASES)
def test_lengths(lib, positions, new, groups, past, H, Hk, D, page, dt):
    """A row past the table's end is NaN; the sequences within it are what they are by the definition."""
    bt = make(positions, new, groups, past, Hk, D, page, dt)
    q = bt.tokens(H)
    ry, rl, by, bl = reference(bt, q, D ** -0.5)       # of the lengths within the table
    for fill in (0, 0xff):
        y, lse = guarded(lib, bt, q, H, fill)
        for b, c in enumerate(new):
            rows = slice(bt.ptr[b], bt.ptr[b] + c)
            if b in past:
                behind = slice(bt.ptr[b] + max(0, c - past[b]), bt.ptr[b] + c)      # rows whose own position has no page
                assert torch.isnan(y[:, behind]).all() and torch.isnan(lse[:, behind]).all(), b
            else:
                R.assert_within(lse[:, rows], rl[:, rows], bl[:, rows], f"lse of {b}")
                R.assert_within(y[:, rows], ry[:, rows], by[:, rows], f"y of {b}")


@pytest.mark.parametrize("H,Hk,D", [(1, 1, 64), (3, 3, 128), (10, 5, 64)])
def test_pointers_that_overlap(lib, H, Hk, D):
    """Nothing is promised about such a call but that it stays within its workspace and ends."""
    bt = Grouped([(600, 1), (500, 1), (512, 1), (300, 1), (450, 1)], [(3, 256), (2, 128)], Hk, D, 16, F16, seed=42)
    q = bt.tokens(H)
    for p in ([0, 5, 0, 5, 0, 5], [5, 0, 5, 0, 5, 0], [-3, 1 << 30, 2, 5, 1, 4]):
        bt.dst_ptr.copy_(torch.tensor(p, dtype=torch.int32))
        guarded(lib, bt, q, H, 0)
