"""The narrow passes of attention behind shared prefixes: every block that is launched has slots of its own in the workspace,
whatever the lengths, of which the host knows nothing."""
import ctypes as C

import pytest

from tests.test_prefix_args import cache
from tests.test_relattn_args import FAKE, b  # noqa: F401

UNITS = 256     # without a device the library plans for as many compute units


def up(n, to):
    return -(-n // to) * to


def needed(num_dst, heads, kv_heads, width, positions, sequences):
    """Bytes of a narrow pass over `sequences` sequences or groups: tiles of 16 rows and 16,384 / width keys.  A launch is a multiple
    of 8 blocks; each leaves up to two states of (width + 2) * 16 floats and four records of 16 bytes."""
    steps = -(-max(positions, 1) // (16384 // width))
    if steps == 1:
        return 0      # nothing is cut
    slots = 2 * up(min((num_dst * heads // kv_heads // 16 + sequences) * kv_heads * steps, 2 * UNITS), 8)
    return up(slots * 16 * (width + 2) * 4, 256) + 2 * slots * 16


@pytest.mark.parametrize("width", [64, 128])
def test_every_launched_block_has_its_slots(b, width):  # noqa: F811
    tried = 0
    for heads, kv_heads in ((1, 1), (2, 1), (3, 3), (4, 2), (6, 6), (32, 4), (5, 5), (16, 16)):
        for batch, num_dst in ((1, 1), (2, 2), (3, 3), (5, 7), (17, 17), (64, 64)):
            for table in (16, 17, 31, 32, 48, 264, 1000):
                for groups in (1, 2, 9):
                    group = heads // kv_heads
                    sequences, shared = min(batch, num_dst), min(groups, num_dst)
                    passes = [n for n in (sequences, shared) if num_dst * group <= 16 * n]
                    rows = num_dst * heads
                    states = 2 * (up(rows * width * 4, 256) + up(rows * 4, 256))
                    need = states + sum(needed(num_dst, heads, kv_heads, width, table * 16, n) for n in passes)
                    p = b._Prefix(groups, FAKE, FAKE)
                    c = cache(b, width=width, kv_heads=kv_heads, batch=batch, table_width=table)
                    have = b.load().tiga_mp_attention_prefix_fwd_workspace(C.byref(c), C.byref(p), num_dst, heads)
                    assert have >= need, (heads, kv_heads, batch, num_dst, table, groups)
                    tried += 1
    assert tried == 8 * 6 * 7 * 3
