"""A group's length past a new token: NaN only where the positions that are read once reach it; the validation goes by the length."""
import pytest
import torch

from tests.test_gpu_prefix_attention import Grouped, compare, run

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


def refused(lib, bt):
    with pytest.raises(lib.TigaError) as e:
        lib.tiga_prefix_validate(bt.cache(lib), bt.num_dst, bt.dst_ptr, bt.group_ptr, bt.group_len)
    assert e.value.code == lib.TIGA_EGRAPH


@pytest.mark.parametrize("new", [1, 30])
def test_right_where_less_is_read_once(lib, new):
    """128 of 200 positions, with a first new token at 150; none of a group of one's."""
    bt = Grouped([(300, new), (150 + new, new), (90, new)], [(2, 150), (1, 60)], 2, 64, 16, BF16, seed=1)
    bt.group_len.copy_(torch.tensor([200, 5000], dtype=torch.int32))
    refused(lib, bt)
    compare(lib, bt, 4, "less than the length")


@pytest.mark.parametrize("first,wrong", [(127, True), (128, False), (129, False)])
def test_the_border(lib, first, wrong):
    bt = Grouped([(300, 1), (first + 1, 1)], [(2, min(first, 200))], 1, 128, 16, BF16, seed=2)
    bt.group_len.fill_(200)
    refused(lib, bt)
    y = run(lib, bt, bt.tokens(2))
    torch.cuda.synchronize()
    assert torch.isfinite(y[:, 0].float()).all() and bool(torch.isnan(y[:, 1]).all()) == wrong
    assert wrong or torch.isfinite(y.float()).all()
