"""Eviction from the longest cache that is accepted: positions up to a group's rounding of 2^31."""
import pytest
import torch

pytestmark = pytest.mark.gpu

F16 = torch.float16


@pytest.mark.parametrize("less", [0, 2048])      # the whole table; the last length whose rounding up fits 31 bits
def test_the_heaviest_positions(lib, less):
    """A table that names 64 pages in turn, one cell of which outweighs the others: it comes every 65,536 positions, and the first
    of them stay, beside the last positions."""
    page, P, D, keep, recent = 1024, 64, 64, 7, 2
    width = (1 << 21) - 2
    n = width * page - less
    g = torch.Generator().manual_seed(91)
    k, v = (torch.randn(P, 1, page, D, generator=g).to(F16).cuda() for _ in range(2))
    w = torch.rand(P, 1, page, generator=g)
    heavy = 40 * page + 77
    w.view(-1)[heavy] = 3.0
    table = (torch.arange(width) % P).to(torch.int32)[None].cuda()
    length = torch.tensor([n], dtype=torch.int32, device="cuda")
    tk, tv, tw = torch.zeros_like(k[:1]), torch.zeros_like(v[:1]), torch.zeros(1, 1, page, device="cuda")
    to = lib.KvCache(tk, tv, torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"))
    kept = torch.full((1, 1, keep), -9, dtype=torch.int32, device="cuda")
    lib.tiga_mp_cache_evict(lib.KvCache(k, v, table, length), w.cuda(), to, tw, keep=keep, recent=recent, kept=kept)
    torch.cuda.synchronize()
    want = [heavy + i * P * page for i in range(keep - recent)] + [n - 2, n - 1]
    assert kept.flatten().tolist() == want and to.length.tolist() == [keep]
    at = torch.tensor(want)
    cells = at // page % P, at % page
    assert torch.equal(tk[0, 0, :keep].cpu(), k.cpu()[cells[0], 0, cells[1]])
    assert torch.equal(tv[0, 0, :keep].cpu(), v.cpu()[cells[0], 0, cells[1]])
    assert torch.equal(tw[0, 0, :keep].cpu(), w[cells[0], 0, cells[1]])
