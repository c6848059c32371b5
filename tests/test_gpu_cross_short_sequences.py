"""Gradients of sequences with few sources do not depend on the padding of their batch, and are as exact as alone."""
import pytest
import torch

from tests import relattn_vjp_ref as V

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16
TILE = {64: 128, 128: 64}


def make(B, H, Hk, N, S, D, dt, sigma=1.0, seed=0):
    g = torch.Generator().manual_seed(seed)
    t = lambda s, *shape: (s * torch.randn(*shape, generator=g)).to(dt).cuda()
    return t(sigma, B, H, N, D), t(sigma, B, Hk, S, D), t(1.0, B, Hk, S, D), t(1.0, B, H, N, D)


def run(lib, q, k, v, dy, lens=None, want=("dq", "dk", "dv")):
    lens = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    y, lse = lib.tiga_mp_attention_cross_fwd(q, k, v, lens, want_lse=True)
    g = lib.tiga_mp_attention_cross_bwd(q, k, v, y, lse, dy, lens, want=want)
    torch.cuda.synchronize()
    return y, lse, g


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dt", [F16, BF16])
@pytest.mark.parametrize("N", [1, 40, 300])
def test_padded_batch(lib, N, D, dt):
    """Peaked weights: where one source has nearly all of a row's weight, ds is small against delta's terms."""
    lens = [700, 2, 3, 5, 1, 0, TILE[D], TILE[D] + 1]
    q, k, v, dy = make(len(lens), 4, 2, N, 700, D, dt, sigma=1.6, seed=N)
    for b, n in enumerate(lens):
        k[b, :, n:], v[b, :, n:] = float("nan"), float("inf")
    y, lse, g = run(lib, q, k, v, dy, lens)
    kz, vz = (torch.nan_to_num(t, nan=0.0, posinf=0.0) for t in (k, v))
    lse = torch.where(torch.isinf(lse), torch.zeros_like(lse), lse)       # of the empty sequence, whose sums are empty
    V.check(g, q, kz, vz, y, lse, dy, D ** -0.5, TILE[D], lens, f"{N, D, dt}")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dt", [F16, BF16])
@pytest.mark.parametrize("n", [1, 2, 5, 64])
def test_alone_and_beside_a_long_one(lib, n, D, dt):
    """The same bits: 30 rows are one streamed tile, so that every sum has the same order in both."""
    q, k, v, dy = make(2, 2, 2, 30, 900, D, dt, seed=n)
    _, _, both = run(lib, q, k, v, dy, [900, n])
    _, _, alone = run(lib, q[1:], k[1:, :, :n], v[1:, :, :n], dy[1:])
    for name in both:
        x = both[name][1:]
        assert torch.equal(x if name == "dq" else x[:, :, :n], alone[name]), name


@pytest.mark.parametrize("N", [30, 1500])
def test_gradients_one_at_a_time(lib, N):
    """Without dq the rows' statistics are the same bits, of short and of long sequences."""
    lens = [500, 3, 64, 0, 129]
    q, k, v, dy = make(len(lens), 4, 2, N, 500, 64, BF16, seed=3)
    _, _, whole = run(lib, q, k, v, dy, lens)
    for name in ("dq", "dk", "dv"):
        _, _, one = run(lib, q, k, v, dy, lens, want=(name,))
        assert list(one) == [name] and torch.equal(one[name], whole[name]), name
