"""Values that are not finite reach the rows that see them, as they are, and nothing else: no row through a weight of 0, and no
row through what fills a tile past the last source."""
import pytest
import torch

from tests.paged_ref import Batch

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16
INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dt", [F16, BF16])
@pytest.mark.parametrize("N,S", [(1, 1), (1, 37), (3, 700), (2, 4001), (40, 5), (300, 65), (130, 129), (70, 1501), (300, 128)])
def test_the_last_source(lib, N, S, D, dt):
    g = torch.Generator().manual_seed(S)
    t = lambda *s: (0.3 * torch.randn(*s, generator=g)).to(dt).cuda()
    q, k, v = t(2, 4, N, D), t(2, 2, S, D), t(2, 2, S, D)
    n = max(1, S // 2)
    lens = torch.tensor([S, n], dtype=torch.int32, device="cuda")
    ref, rl = lib.tiga_mp_attention_cross_fwd(q, k, v, lens, want_lse=True)
    for b, last in enumerate((S - 1, n - 1)):
        v[b, :, last, 3], v[b, :, last, 5], v[b, :, last, 17] = INF, -INF, NAN
        v[b, :, last + 1:] = NAN
    y, lse = lib.tiga_mp_attention_cross_fwd(q, k, v, lens, want_lse=True)
    torch.cuda.synchronize()
    assert bool((y[..., 3] == INF).all()) and bool((y[..., 5] == -INF).all()) and bool(torch.isnan(y[..., 17]).all())
    keep = [d for d in range(D) if d not in (3, 5, 17)]
    assert torch.equal(y[..., keep], ref[..., keep]) and torch.equal(lse, rl)


@pytest.mark.parametrize("dt", [F16, BF16])
@pytest.mark.parametrize("lens", [[(1, 1), (50, 1), (4001, 1)], [(700, 1)], [(100, 1)] * 70])
def test_the_newest_token(lib, lens, dt):
    """Single tokens: the row sees its own value."""
    bt = Batch(lens, 2, 128, 16, dt, seed=1)
    bt.k.mul_(0.3)
    q = 0.3 * bt.tokens(8)
    ref = lib.tiga_mp_attention_paged_fwd(bt.cache(lib), q, bt.dst_ptr)
    for b, (n, _) in enumerate(lens):
        page = int(bt.table[b, (n - 1) // 16])
        bt.v[page, :, (n - 1) % 16, 3] = INF
        bt.v[page, :, (n - 1) % 16 + 1:] = NAN
    y = lib.tiga_mp_attention_paged_fwd(bt.cache(lib), q, bt.dst_ptr)
    torch.cuda.synchronize()
    keep = [d for d in range(128) if d != 3]
    assert bool((y[..., 3] == INF).all()) and torch.equal(y[..., keep], ref[..., keep])
