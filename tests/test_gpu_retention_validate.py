"""A page that two positions' places name is reported before weights are added to it or rows moved over it."""
import pytest
import torch

from tests.paged_ref import Batch
from tests.test_gpu_prefix_attention import Grouped

pytestmark = pytest.mark.gpu

F16 = torch.float16
LENS = [(300, 1), (290, 1), (40, 0), (0, 0), (17, 3)]


def refused(lib, bt, *names):
    with pytest.raises(lib.TigaError) as e:
        lib.tiga_retention_validate(bt.cache(lib))
    assert e.value.code == lib.TIGA_EGRAPH and all(f"sequence {n}" in str(e.value) for n in names), str(e.value)


@pytest.mark.parametrize("page", [1, 16, 512])
def test_pages_of_their_own(lib, page):
    bt = Batch(LENS, 2, 64, page, F16, seed=1)
    lib.tiga_retention_validate(bt.cache(lib))


@pytest.mark.parametrize("copies", [True, False])
def test_a_shared_prefix(lib, copies):
    """In copies; in the same pages, which attention takes and the weights do not."""
    bt = Grouped(LENS, [(2, 256)], 2, 64, 16, F16, copies=copies, seed=2)
    lib.tiga_prefix_validate(bt.cache(lib), bt.num_dst, bt.dst_ptr, bt.group_ptr, bt.group_len)
    if copies:
        lib.tiga_retention_validate(bt.cache(lib))
    else:
        refused(lib, bt, 0, 1)


def test_places(lib):
    bt = Batch(LENS, 1, 64, 16, F16, seed=3)
    table = bt.table.clone()

    def put(b, e, page):
        bt.table.copy_(table)
        bt.table[b, e] = page

    put(4, 1, int(table[2, 2]))            # the last pages that they need
    refused(lib, bt, 2, 4)
    put(0, 18, int(table[0, 3]))           # one sequence, twice
    refused(lib, bt, 0)
    put(2, 3, int(table[0, 3]))            # behind its 40 positions
    lib.tiga_retention_validate(bt.cache(lib))
    put(3, 0, int(table[0, 3]))            # of a sequence without positions
    lib.tiga_retention_validate(bt.cache(lib))
    for bad in (-1, bt.num_pages, 2 ** 31 - 1):
        put(0, 3, bad)
        bt.table[1, 3] = bad               # no page, so no one's
        lib.tiga_retention_validate(bt.cache(lib))
    bt.table.copy_(table)
    bt.length[0] = 1 << 30                 # past the table; negative
    bt.length[2] = -5
    lib.tiga_retention_validate(bt.cache(lib))
