"""binary16 gradients where weights and ds lie below its normal numbers, or above its largest: long flat softmaxes, small and
large cotangents and values.  Against the VJP of the forward's own y and lse in 64 bits (relattn_vjp_ref)."""
import pytest
import torch

from tests import relattn_vjp_ref as V
from tests.test_gpu_cross_short_sequences import TILE, make, run

pytestmark = pytest.mark.gpu

F16 = torch.float16


def check(lib, q, k, v, dy, lens=None, what="", finite=True):
    y, lse, g = run(lib, q, k, v, dy, lens)
    D = q.shape[3]
    if finite:
        assert all(bool(torch.isfinite(t).all()) for t in g.values()), what
    V.check(g, q, k, v, y, torch.where(torch.isinf(lse), torch.zeros_like(lse), lse), dy, D ** -0.5, TILE[D], lens, what)
    return g


@pytest.mark.parametrize("size", [1.0, 1e-2, 1e-3, 1e-4, 1e-5])
@pytest.mark.parametrize("N,S,D", [(257, 8192, 64), (130, 4001, 128), (200, 77, 64), (64, 50, 128), (1, 20000, 64)])
def test_small_cotangents(lib, N, S, D, size):
    q, k, v, dy = make(1, 2, 1, N, S, D, F16, seed=S)
    check(lib, q, k, v, (size * dy.float()).half(), what=f"{N, S, D, size}")


def test_long_flat_softmax(lib):
    """65536 sources of alike weights, 1.5e-5 each."""
    q, k, v, dy = make(1, 1, 1, 33, 65536, 64, F16, sigma=0.1, seed=1)
    for size in (1.0, 1e-3):
        check(lib, q, k, v, (size * dy.float()).half(), what=f"flat {size}")


def test_gradients_that_only_add_up(lib):
    """Every ds is below the smallest binary16 number, and their sum is not: values and keys of one sign pattern."""
    S, D = 16384, 64
    sign = torch.where(torch.arange(S) % 2 == 0, 1.0, -1.0)
    q = torch.zeros(1, 1, 40, D)
    k, v = torch.zeros(1, 1, S, D), torch.zeros(1, 1, S, D)
    k[..., 1], v[..., 0] = sign, sign
    dy = torch.zeros(1, 1, 40, D)
    dy[..., 0] = 2e-4
    q, k, v, dy = (t.half().cuda() for t in (q, k, v, dy))
    g = check(lib, q, k, v, dy, what="coherent")
    # p = 1 / S, dp = dy_0 sign, delta = 0: dq_1 = scale dy_0, which is 2.5e-5, a subnormal number: half a step is 2^-25
    want = float(dy[0, 0, 0, 0]) * D ** -0.5
    off = float((g["dq"][..., 1].double() - want).abs().max())
    assert off <= want * 2.0 ** -10 + 2.0 ** -25 and (g["dq"][..., 2:] == 0).all()


@pytest.mark.parametrize("S", [60, 1500])
def test_rows_of_very_different_cotangents(lib, S):
    """A row's dq is as exact as if it were alone, whatever its neighbours' cotangents; rows without any get 0."""
    q, k, v, dy = make(1, 2, 1, 70, S, 64, F16, seed=2)
    size = (10.0 ** -torch.arange(70).remainder(6)).cuda()
    size[5::10] = 0.0
    dy = (dy.float() * size[:, None]).half()
    g = check(lib, q, k, v, dy, what="rows")
    assert (g["dq"][:, :, 5::10] == 0).all()
    # and a source head of small cotangents beside one of large ones
    q, k, v, dy = make(1, 2, 2, 70, S, 64, F16, seed=3)
    dy[:, 1] = (dy[:, 1].float() * 1e-5).half()
    check(lib, q, k, v, dy, what="heads")


@pytest.mark.parametrize("S", [60, 1500])
@pytest.mark.parametrize("vsize,dsize,ksize", [(5000.0, 5.0, 0.01), (1.0, 5000.0, 0.01), (1e-4, 1e-3, 3.0), (10000.0, 1e-4, 1.0)])
def test_large_and_tiny_values(lib, S, vsize, dsize, ksize):
    """Peaked weights and |dy| |v| past binary16's largest: ds alone would overflow, the gradients of q do not (some of k and v
    do: infinities of the right sign)."""
    q, k, v, dy = make(1, 2, 2, 90, S, 64, F16, seed=4)
    q = q * 4
    k = (k.float() * ksize).half()
    k[:, :, ::7] *= 3
    q = (q.float() / ksize).clamp(-400, 400).half()
    g = check(lib, q, k, (v.float() * vsize).half(), (dy.float() * dsize).half(), what=f"{S, vsize, dsize}", finite=False)
    assert torch.isfinite(g["dq"]).all()


def test_padded_batch(lib):
    lens = [900, 2, 0, 129, 128, 64]
    q, k, v, dy = make(len(lens), 4, 2, 150, 900, 64, F16, seed=5)
    for b, n in enumerate(lens):
        k[b, :, n:], v[b, :, n:] = 0, 0
    dy = (1e-3 * dy.float()).half()
    y, lse, g = run(lib, q, k, v, dy, lens)
    kn, vn = k.clone(), v.clone()
    for b, n in enumerate(lens):
        kn[b, :, n:], vn[b, :, n:] = float("nan"), float("inf")      # what lies in the padding does not count
    _, _, gn = run(lib, q, kn, vn, dy, lens)
    assert all(torch.equal(g[n], gn[n]) for n in g)
    check(lib, q, k, v, dy, lens, what="padded")


def test_captured(lib):
    q, k, v, dy = make(1, 4, 2, 300, 900, 64, F16, seed=7)
    small = (dy.float() * 1e-3).half()
    cur = dy.clone()
    y, lse, _ = run(lib, q, k, v, dy)
    call = lambda: lib.tiga_mp_attention_cross_bwd(q, k, v, y, lse, cur)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for i, d in enumerate((dy, small, small, dy)):
        cur.copy_(d)
        graph.replay()
        ref = call()
        torch.cuda.synchronize()
        assert all(torch.equal(out[n], ref[n]) for n in out), i


@pytest.mark.parametrize("dt", [F16, torch.bfloat16])
@pytest.mark.parametrize("S", [60, 900])
@pytest.mark.parametrize("x", [float("inf"), float("nan")])
def test_a_cotangent_that_is_not_finite(lib, x, S, dt):
    """It stays in its row of dq and in its source head's dk and dv, where it shows (a loss scale's overflow is looked for)."""
    q, k, v, dy = make(1, 4, 2, 100, S, 64, dt, seed=8)
    _, _, a = run(lib, q, k, v, dy)
    dy[0, 1, 37, 11] = x
    _, _, b = run(lib, q, k, v, dy)
    keep = torch.ones(4, 100, dtype=torch.bool, device="cuda")
    keep[1, 37] = False
    assert torch.equal(b["dq"][0][keep], a["dq"][0][keep]) and not bool(torch.isfinite(b["dq"][0, 1, 37]).any())
    for name in ("dk", "dv"):
        assert torch.equal(b[name][0, 1], a[name][0, 1])
    assert not bool(torch.isfinite(b["dk"][0, 0]).any()) and not bool(torch.isfinite(b["dv"][0, 0, :, 11]).any())
