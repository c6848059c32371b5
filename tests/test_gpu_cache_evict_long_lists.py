"""Eviction to budgets as large as 32 bits count: far more than there are positions."""
import pytest
import torch

from tests.test_gpu_cache_evict import Case, same

pytestmark = pytest.mark.gpu

F16 = torch.float16


@pytest.mark.parametrize("n", [300, 40_000])       # a block for the list, and several
@pytest.mark.parametrize("keep", [2 ** 31 - 1, 2 ** 31 - 1024])
def test_all_positions_stay(lib, n, keep):
    c = Case([n], 1, 64, 64, F16, n, 5, seed=81)
    _, k, v, w = c.expected()
    to = c.to.cache(lib)
    torch.cuda.empty_cache()
    kept = torch.full((1, 1, keep), -9, dtype=torch.int32, device="cuda")
    lib.tiga_mp_cache_evict(c.bt.cache(lib), c.weights, to, c.to_weights, keep=keep, recent=5, kept=kept)
    torch.cuda.synchronize()
    assert torch.equal(kept[0, 0, :n].cpu(), torch.arange(n, dtype=torch.int32))
    for part in kept[0, 0, n:].split(1 << 28):
        assert (part == -1).all()
    assert same(c.to.k, k) and same(c.to.v, v) and same(c.to_weights, w) and to.length.tolist() == [n]
    del kept
    torch.cuda.empty_cache()
