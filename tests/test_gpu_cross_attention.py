"""Cross attention (forward and VJP) against 64 bits on the CPU; the bounds are derived in relattn_ref."""
import pytest
import torch

from tests import relattn_ref as R

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


def make(B, H, Hk, N, S, D, dt, seed=0, sigma=1.0):
    g = torch.Generator().manual_seed(seed)
    t = lambda *s: (sigma * torch.randn(*s, generator=g)).to(dt).cuda()
    return t(B, H, N, D), t(B, Hk, S, D), t(B, Hk, S, D), torch.randn(B, H, N, D, generator=g).to(dt).cuda()


def both(lib, q, k, v, dy, lens=None, scale=None, layout="bhnd"):
    y, lse = lib.tiga_mp_attention_cross_fwd(q, k, v, lens, scale, want_lse=True, layout=layout)
    g = lib.tiga_mp_attention_cross_bwd(q, k, v, y, lse, dy, lens, scale, layout=layout)
    torch.cuda.synchronize()
    return dict(y=y, lse=lse, **g)


def compare(lib, q, k, v, dy, lens=None, scale=None, what=""):
    got = both(lib, q, k, v, dy, lens, scale)
    ref, bound = R.cross(q, k, v, lens, q.shape[3] ** -0.5 if scale is None else scale, dy)
    for name in ("lse", "y", "dv", "dq", "dk"):
        R.assert_within(got[name], ref[name], bound[name], f"{what} {name}")


# batch, heads, source heads, destinations, sources, width, type: lengths around 1, 16, 32, 64 and 128, odd ones,
# few rows over many sources and many rows over few, shared heads
CASES = [
    (1, 1, 1, 1, 1, 64, F16), (2, 2, 1, 1, 17, 128, BF16), (1, 3, 3, 2, 64, 64, BF16), (3, 4, 2, 16, 65, 128, F16),
    (1, 8, 1, 31, 127, 64, F16), (2, 6, 2, 33, 128, 128, BF16), (1, 2, 2, 64, 33, 128, F16), (2, 4, 4, 129, 129, 64, BF16),
    (1, 4, 1, 300, 77, 64, F16), (1, 1, 1, 1, 3001, 128, F16), (2, 16, 2, 1, 1500, 64, BF16), (1, 5, 1, 7, 1000, 128, BF16),
    (1, 2, 1, 1025, 9, 64, BF16), (1, 2, 2, 513, 511, 128, F16), (1, 3, 1, 200, 1, 128, BF16), (1, 2, 1, 2000, 40, 128, F16),
    (2, 1, 1, 130, 2050, 64, F16), (17, 1, 1, 3, 5, 64, BF16),
]


@pytest.mark.parametrize("B,H,Hk,N,S,D,dt", CASES)
def test_against_64_bits(lib, B, H, Hk, N, S, D, dt):
    q, k, v, dy = make(B, H, Hk, N, S, D, dt, seed=N + S)
    compare(lib, q, k, v, dy, what=f"{(B, H, Hk, N, S, D, dt)}")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dt", [F16, BF16])
@pytest.mark.parametrize("N,S", [(1, 300), (70, 300), (300, 70)])
def test_padded_batch(lib, N, S, D, dt):
    """Lengths of 0, 1, the whole and beyond; what lies in the padding (NaN, infinities) is never seen."""
    q, k, v, dy = make(6, 4, 2, N, S, D, dt, seed=3)
    lens = torch.tensor([S, 0, 1, S // 2, S + 5, -3], dtype=torch.int32, device="cuda")
    for b, n in enumerate(lens.tolist()):
        n = max(0, min(S, n))
        k[b, :, n:], v[b, :, n:] = float("nan"), float("inf")
    got = both(lib, q, k, v, dy, lens)
    kc, vc = k.clone(), v.clone()
    for b, n in enumerate(lens.tolist()):
        n = max(0, min(S, n))
        kc[b, :, n:], vc[b, :, n:] = 0, 0
    ref, bound = R.cross(q, kc, vc, lens, D ** -0.5, dy)
    for name in ("lse", "y", "dv", "dq", "dk"):
        R.assert_within(got[name], ref[name], bound[name], name)
    assert (got["y"][1] == 0).all() and torch.isneginf(got["lse"][1]).all() and (got["dq"][1] == 0).all()


@pytest.mark.parametrize("dt", [F16, BF16])
@pytest.mark.parametrize("N", [1, 100])
def test_large_and_rising_scores(lib, dt, N):
    """Scores over about +-60, and scores that grow along the sources, so that the reference point keeps moving."""
    q, k, v, dy = make(1, 2, 1, N, 700, 128, dt, seed=5, sigma=2.5)
    compare(lib, q, k, v, dy, what="large")
    k = (torch.linspace(-1.5, 1.5, 700)[None, None, :, None] + 0.01 * k.float().cpu()).to(dt).cuda()
    compare(lib, torch.ones_like(q), k, v, dy, what="rising")
    compare(lib, torch.ones_like(q), k.flip(2).contiguous(), v, dy, what="falling")


def test_lowest_values(lib):
    """Keys that give scores of the type's lowest order for all but one source: its value comes back."""
    q, k, v, dy = make(1, 1, 1, 40, 200, 64, BF16, seed=6)
    q[:], k[:] = 1.0, -3.0e38
    k[0, 0, 77] = 0.25
    y, lse = lib.tiga_mp_attention_cross_fwd(q, k, v, want_lse=True)
    torch.cuda.synchronize()
    assert torch.equal(y, v[:, :, 77:78].expand_as(y)) and torch.isfinite(lse).all()


def test_scale_given(lib):
    q, k, v, dy = make(1, 2, 2, 50, 60, 64, F16, seed=7)
    compare(lib, q, k, v, dy, scale=0.031, what="scale")


def test_layouts_and_strides_give_the_same_bits(lib):
    """Rows before heads, slices of a joint projection, sources shared by the batch (a stride of 0)."""
    B, H, Hk, N, S, D = 2, 4, 2, 70, 90, 64
    g = torch.Generator().manual_seed(8)
    kv = torch.randn(1, S, 2, Hk, D, generator=g).to(BF16).cuda().expand(B, -1, -1, -1, -1)
    qx = torch.randn(B, N, H, 3 * D, generator=g).to(BF16).cuda()[..., D:2 * D]
    dy = torch.randn(B, N, H, D, generator=g).to(BF16).cuda()
    k, v = kv[:, :, 0], kv[:, :, 1]
    a = both(lib, qx, k, v, dy, layout="bnhd")
    h = lambda t: t.permute(0, 2, 1, 3).contiguous()
    b = both(lib, h(qx), h(k), h(v), h(dy))
    for name in b:
        x = a[name] if name == "lse" else h(a[name])
        assert torch.equal(x, b[name]), name


def test_gradients_one_at_a_time_are_the_same_bits(lib):
    q, k, v, dy = make(2, 4, 2, 150, 260, 128, BF16, seed=9)
    y, lse = lib.tiga_mp_attention_cross_fwd(q, k, v, want_lse=True)
    whole = lib.tiga_mp_attention_cross_bwd(q, k, v, y, lse, dy)
    for name in ("dq", "dk", "dv"):
        one = lib.tiga_mp_attention_cross_bwd(q, k, v, y, lse, dy, want=(name,))
        assert list(one) == [name] and torch.equal(one[name], whole[name])


@pytest.mark.parametrize("N,S", [(1, 4000), (333, 777), (3000, 50)])
def test_repeated_calls_are_bit_identical(lib, N, S):
    q, k, v, dy = make(2, 4, 2, N, S, 64, F16, seed=10)
    a, b = both(lib, q, k, v, dy), both(lib, q, k, v, dy)
    for name in a:
        assert torch.equal(a[name], b[name]), name


def test_empty_sizes(lib):
    q, k, v, dy = make(2, 4, 2, 5, 7, 64, F16)
    y, lse = lib.tiga_mp_attention_cross_fwd(q, k[:, :, :0], v[:, :, :0], want_lse=True)
    assert (y == 0).all() and torch.isneginf(lse).all()
    g = lib.tiga_mp_attention_cross_bwd(q, k[:, :, :0], v[:, :, :0], y, lse, dy)
    assert (g["dq"] == 0).all() and g["dk"].shape == (2, 2, 0, 64)
    y, lse = lib.tiga_mp_attention_cross_fwd(q[:, :, :0], k, v, want_lse=True)
    g = lib.tiga_mp_attention_cross_bwd(q[:, :, :0], k, v, y, lse, y)
    assert y.shape == (2, 4, 0, 64) and (g["dk"] == 0).all() and (g["dv"] == 0).all()


def test_autograd_matches_differences(lib):
    """The gradient of a scalar of y along a random direction against a central difference of the 64-bit forward."""
    q, k, v, dy = make(1, 4, 2, 20, 33, 64, F16, seed=11)
    for t in (q, k, v):
        t.requires_grad_(True)
    y = lib.cross_attention(q, k, v)
    y.backward(dy)
    gen = torch.Generator().manual_seed(1)
    for t, name in ((q, "q"), (k, "k"), (v, "v")):
        d = torch.randn(t.shape, generator=gen, dtype=torch.float64)
        h = 1e-4

        def loss(sign):
            a = dict(q=q.detach().double().cpu(), k=k.detach().double().cpu(), v=v.detach().double().cpu())
            a[name] = a[name] + sign * h * d
            total = 0.0
            for i in range(4):
                p = torch.softmax(a["q"][0, i] @ a["k"][0, i // 2].t() * 64 ** -0.5, 1)
                total = total + (p @ a["v"][0, i // 2] * dy[0, i].double().cpu()).sum()
            return total

        num = (loss(1.0) - loss(-1.0)) / (2 * h)
        ref, bound = R.cross(q, k, v, None, 64 ** -0.5, dy)
        tol = (bound["d" + name] * d.abs()).sum() + 1e-6 * (1 + abs(num))    # the difference itself: O(h^2)
        assert abs((t.grad.double().cpu() * d).sum() - num) <= tol


def test_autograd_broadcast_cotangent_and_frozen_inputs(lib):
    q, k, v, _ = make(2, 2, 1, 10, 20, 64, BF16, seed=12)
    k.requires_grad_(True)
    lib.cross_attention(q, k, v).sum().backward()
    assert q.grad is None and k.grad.shape == k.shape
    y, lse = lib.tiga_mp_attention_cross_fwd(q, k.detach(), v, want_lse=True)
    g = lib.tiga_mp_attention_cross_bwd(q, k.detach(), v, y, lse, torch.ones_like(y), want=("dk",))
    assert torch.equal(k.grad, g["dk"])


@pytest.mark.parametrize("N,S", [(1, 2000), (200, 300)])
def test_captured_and_replayed(lib, N, S):
    """Forward and backward in a graph, replayed with new inputs and eager work in between."""
    lens = torch.tensor([S, S // 3], dtype=torch.int32, device="cuda")
    sets = [make(2, 4, 2, N, S, 64, BF16, seed=20 + i) for i in range(3)]
    ins = [t.clone() for t in sets[0]]
    step = lambda q, k, v, dy: both_async(lib, q, k, v, dy, lens)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*ins)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(*ins)
    for i in range(4):
        for a, b in zip(ins, sets[i % 3]):
            a.copy_(b)
        lens.copy_(torch.tensor([S, [S // 3, 0, 1, S][i]], dtype=torch.int32))
        graph.replay()
        ref = step(*sets[i % 3])
        torch.cuda.synchronize()
        for name in ref:
            assert torch.equal(out[name], ref[name]), (i, name)


def both_async(lib, q, k, v, dy, lens):
    y, lse = lib.tiga_mp_attention_cross_fwd(q, k, v, lens, want_lse=True)
    return dict(y=y, lse=lse, **lib.tiga_mp_attention_cross_bwd(q, k, v, y, lse, dy, lens))


def test_two_streams_at_once(lib):
    """Two calls in flight, each with its own workspace."""
    a, b = make(2, 4, 2, 300, 900, 128, F16, seed=30), make(1, 8, 1, 1, 5000, 64, BF16, seed=31)
    ra, rb = both(lib, *a), both(lib, *b)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(s1):
            ga = both_async(lib, *a, None)
        with torch.cuda.stream(s2):
            gb = both_async(lib, *b, None)
        torch.cuda.synchronize()
        for name in ra:
            assert torch.equal(ga[name], ra[name]) and torch.equal(gb[name], rb[name]), name


def test_outputs_are_written_inside_their_rows_only(lib):
    """y into the middle of a larger buffer through the C entry point: the guard around it keeps its values."""
    import ctypes as C
    q, k, v, _ = make(2, 2, 2, 37, 50, 64, F16, seed=13)
    buf = torch.full((2, 2, 39, 80), 7.0, dtype=F16, device="cuda")
    L = lib.load()
    rel, qv, kv, vv, _ = lib._cross(q, k, v, None, "bhnd")
    yv = lib._View(buf.data_ptr() + 2 * (80 + 8), *buf.stride()[:3])
    ws = lib._workspace(L.tiga_mp_attention_cross_fwd_workspace(C.byref(rel)), q.device)
    rc = L.tiga_mp_attention_cross_fwd(C.byref(rel), C.byref(qv), C.byref(kv), C.byref(vv), 0.125, C.byref(yv), None,
                                       lib._ptr(ws), ws.numel(), lib._stream())
    assert rc == lib.TIGA_OK
    ref = lib.tiga_mp_attention_cross_fwd(q, k, v, scale=0.125)
    torch.cuda.synchronize()
    assert torch.equal(buf[:, :, 1:38, 8:72], ref)
    buf[:, :, 1:38, 8:72] = 7.0
    assert (buf == 7.0).all()
