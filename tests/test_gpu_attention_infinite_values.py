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


@pytest.mark.parametrize("D,H,Hk", [(64, 2, 2), (128, 4, 1)])
@pytest.mark.parametrize("dt", [F16, BF16])
@pytest.mark.parametrize("lens", [[(40, 40)], [(5, 5), (3, 3)], [(700, 300), (90, 1), (200, 130)], [(129, 129)], [(1500, 3), (20, 2)],
                                  [(4100, 20)], [(2048, 2048)]])
def test_later_tokens_do_not_reach_earlier_ones(lib, lens, dt, D, H, Hk):
    """Infinite and NaN values of some new tokens: rows before them keep their bits, rows from them on have the infinity."""
    bt = Batch(lens, Hk, D, 16, dt, seed=3)
    bt.k.mul_(0.3)
    q = 0.3 * bt.tokens(H)
    ref, rl = lib.tiga_mp_attention_paged_fwd(bt.cache(lib), q, bt.dst_ptr, want_lse=True)
    bad = []                                                  # sequence, token, width, value
    for b, (n, c) in enumerate(lens):
        for t, d, x in ((c - 1, 3, INF), (c // 2, 5, -INF), (c // 3, 17, NAN), (c // 3, 40, INF)):
            bad.append((b, t, d, x))
            p = n - c + t
            bt.v[int(bt.table[b, p // 16]), :, p % 16, d] = x
    y, lse = lib.tiga_mp_attention_paged_fwd(bt.cache(lib), q, bt.dst_ptr, want_lse=True)
    torch.cuda.synchronize()
    assert torch.equal(lse, rl)
    want = ref.clone()
    for b, t, d, x in bad:
        want[:, bt.ptr[b] + t:bt.ptr[b + 1], d] = x
    assert torch.equal(torch.isnan(y), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(y, nan=1.0), torch.nan_to_num(want, nan=1.0))


def test_all_values_of_a_token(lib):
    """A whole row of NaN (a token whose forward broke), keys and values: only it and what follows is NaN.  The NaN scores of
    the later rows move the wavefront's reference points, so earlier rows may round otherwise: either result is off by at
    most u for the weights, u for the output and 2^-12 for fp32 (scores of order 1), of values of at most max|v|."""
    bt = Batch([(300, 200)], 1, 128, 16, BF16, seed=4)
    q = bt.tokens(8)
    ref = lib.tiga_mp_attention_paged_fwd(bt.cache(lib), q, bt.dst_ptr)
    bt.v[int(bt.table[0, 250 // 16]), :, 250 % 16] = NAN
    bt.k[int(bt.table[0, 250 // 16]), :, 250 % 16] = NAN
    y = lib.tiga_mp_attention_paged_fwd(bt.cache(lib), q, bt.dst_ptr)
    torch.cuda.synchronize()
    assert bool(torch.isnan(y[:, 150:]).all())
    top = torch.nan_to_num(bt.v.float()).abs().max()
    assert (y[:, :150].float() - ref[:, :150].float()).abs().max() <= 2 * (2 * 2.0 ** -8 + 2.0 ** -12) * top
