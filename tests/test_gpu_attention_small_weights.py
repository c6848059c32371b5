"""Weights far below the largest of their row: a token that nearly all weight goes to, whose value says nothing, before a long
context that says all.  Each weight enters the value product rounded: u of it; in binary16 at least 2^-25 of an operand that
is at least 2^10 for the row's largest weight, so 2^-35 of that one.  The mass is of unrounded weights; scores, exponentials
and sums are fp32 (relattn_ref)."""
import pytest
import torch

from tests import relattn_ref as R
from tests.paged_ref import Batch

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


def check(y, q, k, v, scale, dt, what):
    """y, q [n, D], k, v [m, D]."""
    q, k, v = (t.double().cpu() for t in (q, k, v))
    f = R.rows(q, k, v, torch.ones(q.shape[0], k.shape[0], dtype=torch.bool), scale)
    top = f["p"].amax(1, keepdim=True)
    loose = f["y_bound"](BF16) if dt == BF16 else None
    u = R.U[dt]
    worst = f["es"].amax(1, keepdim=True)
    # roundings of the weights and of the output, the scores' errors in the weights and in the mass, the sums
    bound = (2 * u + 2 * worst + 2 * R.sums(k.shape[0])) * (f["p"] @ v.abs())
    if dt == F16:
        bound = bound + 2.0 ** -35 * top * v.abs().sum(0) + 2.0 ** -24
    else:
        bound = loose
    R.assert_within(y, f["y"], bound, what)


def context(S, D, gap, dt, seed, spread=0.0):
    """Keys of which the first has a score `gap` above the others' 0 (plus spread), and a value of 0."""
    g = torch.Generator().manual_seed(seed)
    k = spread * torch.randn(S, D, generator=g)
    k[:, 0] = 0.0
    k[0] = 0.0
    k[0, 0] = gap * D ** 0.5 / 4.0
    v = 1.0 + 0.25 * torch.randn(S, D, generator=g)
    v[0] = 0.0
    return k.to(dt), v.to(dt)


def queries(n, D, dt, seed):
    q = torch.randn(n, D, generator=torch.Generator().manual_seed(seed))
    q[:, 0] = 4.0
    return q.to(dt)


@pytest.mark.parametrize("dt", [F16, BF16])
@pytest.mark.parametrize("N,S,D,gap,spread", [(1, 131072, 64, 17.0, 0.0), (40, 20000, 64, 17.0, 0.0), (200, 6000, 128, 15.0, 0.5),
                                              (1, 50000, 128, 16.0, 0.5), (130, 300, 128, 12.0, 0.2), (16, 100, 64, 17.0, 0.0)])
def test_a_heavy_first_source(lib, N, S, D, gap, spread, dt):
    k, v = context(S, D, gap, dt, N, spread)
    q = queries(N, D, dt, S)
    c = lambda t: t[None, None].cuda()
    for what, kk, vv in (("first", k, v), ("last", k.flip(0).contiguous(), v.flip(0).contiguous())):
        y = lib.tiga_mp_attention_cross_fwd(c(q), c(kk), c(vv))
        check(y[0, 0], q, kk, vv, D ** -0.5, dt, f"{what} {N, S, D}")


@pytest.mark.parametrize("new", [1, 30])
def test_paged(lib, new):
    n, D = 30000, 128
    bt = Batch([(n, new)], 1, D, 16, F16, seed=5)
    k, v = context(n, D, 17.0, F16, 3)
    ids = bt.table[0, : -(-n // 16)].long()
    pad = lambda t: torch.cat([t, t.new_zeros(-n % 16, D)]).view(-1, 16, D)[:, None].cuda()
    bt.k[ids], bt.v[ids] = pad(k), pad(v)
    q = queries(new, D, F16, 9)
    y = lib.tiga_mp_attention_paged_fwd(bt.cache(lib), q[None].cuda(), bt.dst_ptr)
    for t in (0, new - 1):
        m = n - new + t + 1
        check(y[0, t:t + 1], q[t:t + 1], k[:m], v[:m], D ** -0.5, F16, f"token {t}")
