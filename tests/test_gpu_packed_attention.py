"""Causal attention of packed sequences against 64 bits on the CPU; the bounds are derived in relattn_ref."""
import pytest
import torch

from tests import relattn_ref as R
from tests.packed_ref import Packed, check, reference

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16

# lengths, heads, source heads, width, type
CASES = [
    ([1], 1, 1, 64, F16),
    ([2], 2, 1, 128, BF16),
    ([1, 1, 1, 1, 1], 4, 2, 64, BF16),
    ([5, 17, 16, 33], 4, 2, 128, F16),
    ([0, 40, 0, 129, 0], 3, 3, 64, F16),
    ([128], 1, 1, 128, BF16),
    ([127, 129], 2, 2, 64, F16),
    ([64, 65, 63], 8, 1, 128, BF16),
    ([256, 1, 31], 2, 1, 128, F16),
    ([300, 7], 6, 2, 64, BF16),
    ([513], 5, 1, 64, F16),
    ([700, 3, 130], 3, 1, 128, BF16),
    ([1300], 1, 1, 128, F16),
    ([1100, 90], 2, 1, 64, BF16),
    ([1 + 7 * (i % 11) for i in range(70)], 2, 2, 64, F16),
    ([3 + (i * 37) % 50 for i in range(150)], 1, 1, 128, BF16),
    ([257] * 3, 32, 2, 64, F16),
    ([140, 20], 16, 16, 128, BF16),
    # long sequences of few heads, whose backward is cut into parts
    ([1500, 300], 2, 1, 128, BF16),
    ([40, 3000], 1, 1, 64, F16),
    ([2600], 4, 1, 64, BF16),
    ([700, 1, 2200], 3, 3, 128, F16),
]


@pytest.mark.parametrize("lens,H,Hk,D,dt", CASES)
def test_against_64_bits(lib, lens, H, Hk, D, dt):
    check(lib, Packed(lens, H, Hk, D, dt, seed=len(lens) + D), f"{(len(lens), lens[0], H, Hk, D)}")


@pytest.mark.parametrize("D,dt", [(64, F16), (128, BF16)])
@pytest.mark.parametrize("scale", [0.02, 0.9])
def test_scales(lib, D, dt, scale):
    check(lib, Packed([200, 70], 2, 1, D, dt, seed=3), "scale", scale=scale)


@pytest.mark.parametrize("lens", [[90, 200], [5, 9], []])
@pytest.mark.parametrize("H,Hk,D,dt", [(4, 2, 64, F16), (2, 2, 128, BF16)])
def test_rows_of_no_sequence(lib, lens, H, Hk, D, dt):
    """They may hold anything, and give 0."""
    s = Packed(lens, H, Hk, D, dt, seed=5, lead=13, tail=150)
    ref = reference(s, D ** -0.5)
    out = s.outside().cuda()
    for t, bad in ((s.q, float("nan")), (s.k, float("inf")), (s.v, float("nan")), (s.dy, float("-inf"))):
        t[:, out] = bad
    check(lib, s, "outside", ref=ref)


@pytest.mark.parametrize("H,Hk", [(4, 2), (6, 1)])
def test_layouts_and_strides(lib, H, Hk):
    """Rows first, all three side by side: the same bits as from tensors of their own."""
    s = Packed([150, 33], H, Hk, 64, BF16, seed=6)
    y, lse = lib.tiga_mp_attention_packed_fwd(s.q, s.k, s.v, s.ptr_t, want_lse=True)
    g = lib.tiga_mp_attention_packed_bwd(s.q, s.k, s.v, y, lse, s.dy, s.ptr_t)
    qkv = torch.cat([s.q, s.k, s.v]).permute(1, 0, 2).contiguous()
    q, k, v = qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:]
    y2, lse2 = lib.tiga_mp_attention_packed_fwd(q, k, v, s.ptr_t, want_lse=True, layout="nhd")
    dy = s.dy.permute(1, 0, 2).contiguous()
    g2 = lib.tiga_mp_attention_packed_bwd(q, k, v, y2, lse2, dy, s.ptr_t, layout="nhd")
    torch.cuda.synchronize()
    assert torch.equal(y2.permute(1, 0, 2), y) and torch.equal(lse, lse2)
    for n in g:
        assert torch.equal(g2[n].permute(1, 0, 2), g[n]), n


def test_each_gradient_alone(lib):
    s = Packed([150, 300], 4, 2, 64, F16, seed=7)
    y, lse = lib.tiga_mp_attention_packed_fwd(s.q, s.k, s.v, s.ptr_t, want_lse=True)
    every = lib.tiga_mp_attention_packed_bwd(s.q, s.k, s.v, y, lse, s.dy, s.ptr_t)
    for want in (("dq",), ("dk",), ("dv",), ("dq", "dv"), ("dk", "dv"), ()):
        g = lib.tiga_mp_attention_packed_bwd(s.q, s.k, s.v, y, lse, s.dy, s.ptr_t, want=want)
        torch.cuda.synchronize()
        assert set(g) == set(want) and all(torch.equal(g[n], every[n]) for n in want), want


def test_a_sequence_does_not_depend_on_the_batch(lib):
    """Alone or among others: the same bits, where no part is split otherwise."""
    s = Packed([90, 400, 33], 2, 2, 64, F16, seed=8)
    y, lse = lib.tiga_mp_attention_packed_fwd(s.q, s.k, s.v, s.ptr_t, want_lse=True)
    g = lib.tiga_mp_attention_packed_bwd(s.q, s.k, s.v, y, lse, s.dy, s.ptr_t)
    one = slice(s.ptr[1], s.ptr[2])
    q, k, v, dy, y1 = (t[:, one].contiguous() for t in (s.q, s.k, s.v, s.dy, y))
    ptr = torch.tensor([0, 400], dtype=torch.int32, device="cuda")
    g1 = lib.tiga_mp_attention_packed_bwd(q, k, v, y1, lse[:, one].contiguous(), dy, ptr)
    torch.cuda.synchronize()
    for n in g:
        assert torch.equal(g[n][:, one], g1[n]), n


BAD = [float("inf"), float("-inf"), float("nan")]


@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("at", [0, 40, 200, 299])
@pytest.mark.parametrize("D,H,Hk,dt", [(64, 2, 1, F16), (128, 1, 1, BF16)])
def test_what_is_not_finite_reaches_nothing_before_it(lib, bad, at, D, H, Hk, dt):
    """Row `at` of the second sequence: forward results before it, and gradients that do not depend on it, are those without
    it (within the bounds: rows that share a wavefront share the steps of their weights' reference points, so a row that is
    NaN may round its neighbours' weights against another point)."""
    s = Packed([20, 300, 40], H, Hk, D, dt, seed=9)
    out, bound = reference(s, D ** -0.5)
    row = s.ptr[1] + at
    before = list(range(s.ptr[1])) + list(range(s.ptr[2], s.N))
    clean = before + list(range(s.ptr[1], row))          # rows that do not see row `at`
    after = before + list(range(row + 1, s.ptr[2]))      # keys that row `at` does not see
    other = before + [r for r in range(s.ptr[1], s.ptr[2]) if r != row]
    for name in ("q", "k", "v", "dy"):
        t = getattr(s, name)
        kept = t[:, row].clone()
        t[0, row, 5] = bad
        y, lse = lib.tiga_mp_attention_packed_fwd(s.q, s.k, s.v, s.ptr_t, want_lse=True)
        g = lib.tiga_mp_attention_packed_bwd(s.q, s.k, s.v, y, lse, s.dy, s.ptr_t)
        torch.cuda.synchronize()
        t[:, row] = kept

        def right(n, got, rows):
            R.assert_within(got[:, rows], out[n][:, rows], bound[n][:, rows], f"{name}: {n}")

        right("y", y, clean)
        right("lse", lse, clean)
        if name in ("q", "dy"):  # its own row alone, and the keys that it sees
            right("dq", g["dq"], other)
            right("dk", g["dk"], after)
            right("dv", g["dv"], after)
            if name == "dy":
                assert not torch.isfinite(g["dv"][0, s.ptr[1]:row + 1, 5]).any()
            assert not torch.isfinite(g["dk"][0, s.ptr[1]:row + 1, 5]).any(), name
        else:  # the rows from it on
            right("dq", g["dq"], clean)
            # an infinite key may have a score of -inf, and so a weight of 0: then only ds * k is not finite, in element 5
            assert not torch.isfinite(g["dq"][0, row:s.ptr[2], 5]).any(), name


def autograd_in_64_bits(s, scale):
    leaves = [t.detach().double().cpu().requires_grad_(True) for t in (s.q, s.k, s.v)]
    g = s.H // s.Hk
    ys = []
    for a, e in zip(s.ptr, s.ptr[1:]):
        q, k, v = (t[:, a:e] for t in leaves)
        k, v = k.repeat_interleave(g, 0), v.repeat_interleave(g, 0)
        sc = (q @ k.transpose(1, 2) * scale).masked_fill(torch.ones(e - a, e - a, dtype=torch.bool).triu(1), -torch.inf)
        ys.append(torch.softmax(sc, -1) @ v)
    return torch.autograd.grad(torch.cat(ys, 1), leaves, s.dy.double().cpu())


def test_autograd_and_differences(lib):
    """The differentiable function gives the VJP's bits, those agree with automatic differentiation in 64 bits, and that
    with central differences of the definition."""
    s = Packed([33, 70], 4, 2, 64, F16, seed=11)
    scale = 64 ** -0.5
    y0, lse = lib.tiga_mp_attention_packed_fwd(s.q, s.k, s.v, s.ptr_t, want_lse=True)
    g0 = lib.tiga_mp_attention_packed_bwd(s.q, s.k, s.v, y0, lse, s.dy, s.ptr_t)
    leaves = [t.clone().requires_grad_(True) for t in (s.q, s.k, s.v)]
    y = lib.packed_attention(*leaves, s.ptr_t)
    g = torch.autograd.grad(y, leaves, s.dy)
    torch.cuda.synchronize()
    assert torch.equal(y, y0)
    out, bound = reference(s, scale)
    for n, a, e in zip(("dq", "dk", "dv"), g, autograd_in_64_bits(s, scale)):
        assert torch.equal(a, g0[n]), n
        R.assert_within(a, e, bound[n], n)
        R.assert_within(out[n], e, 1e-9 * (1 + e.abs()), "the formula's " + n)

    def loss(q, k, v):
        t = Packed.__new__(Packed)
        t.__dict__.update(s.__dict__, q=q, k=k, v=v)
        return (reference(t, scale, False)[0]["y"] * s.dy.double().cpu()).sum()

    base = [t.double().cpu() for t in (s.q, s.k, s.v)]
    for i, n in enumerate(("dq", "dk", "dv")):
        step = torch.zeros_like(base[i])
        step[1, 40, 7], step[0, 2, 3], step[1, 33, 1] = 1.0, -0.5, 2.0
        eps = 1e-4
        moved = [[b + (sign * eps * step if j == i else 0) for j, b in enumerate(base)] for sign in (1, -1)]
        rate = (loss(*moved[0]) - loss(*moved[1])) / (2 * eps)
        assert abs(float(rate) - float((out[n] * step).sum())) < 1e-6 * (1 + abs(float(rate))), n


def test_needs_and_strided_cotangents(lib):
    s = Packed([60, 9], 2, 1, 64, BF16, seed=12)
    q, k, v = s.q.clone().requires_grad_(True), s.k, s.v.clone().requires_grad_(True)
    y = lib.packed_attention(q, k, v, s.ptr_t)
    (y.float().transpose(1, 2) * 2.0).sum().backward()    # an expanded cotangent
    assert q.grad is not None and v.grad is not None and torch.isfinite(q.grad.float()).all()


def test_captured(lib):
    """Lengths that change between replays; eager work in between."""
    s = Packed([900, 2300, 50], 4, 2, 64, BF16, seed=13)
    sides = [s.ptr, [0, 7, 7, 3250], [0, 1, 3250, 3250], [0, 1000, 2000, 3000], [100, 200, 3000, 3100]]
    run = lambda: (lambda y, lse: (y, lse, lib.tiga_mp_attention_packed_bwd(s.q, s.k, s.v, y, lse, s.dy, s.ptr_t)))(
        *lib.tiga_mp_attention_packed_fwd(s.q, s.k, s.v, s.ptr_t, want_lse=True))
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, lse, g = run()
    for p in sides + sides[::-1]:
        s.ptr_t.copy_(torch.tensor(p, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        y2, lse2, g2 = run()
        torch.cuda.synchronize()
        assert torch.equal(y, y2) and torch.equal(lse, lse2) and all(torch.equal(g[n], g2[n]) for n in g)


def test_on_another_stream(lib):
    s = Packed([100, 300], 4, 2, 128, BF16, seed=14)
    y = lib.tiga_mp_attention_packed_fwd(s.q, s.k, s.v, s.ptr_t)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y2 = lib.tiga_mp_attention_packed_fwd(s.q, s.k, s.v, s.ptr_t)
    side.synchronize()
    assert torch.equal(y, y2)


def test_pointers_that_run_backwards_stay_inside(lib):
    """Nothing is promised about such a call but that it stays within the tensors and ends."""
    s = Packed([100, 60, 40], 2, 1, 64, F16, seed=15)
    many = [(i * 7919) % 211 for i in range(200)]
    for p in ([0, 160, 100, 200], [-5, 100, 50, 1 << 30], [200, 100, 50, 0], [1 << 30, -1, 1 << 30, 3], [0, 200] * 30, many,
              [0, 200] * 100):
        ptr = torch.tensor(p, dtype=torch.int32, device="cuda")
        y, lse = lib.tiga_mp_attention_packed_fwd(s.q, s.k, s.v, ptr, want_lse=True)
        lib.tiga_mp_attention_packed_bwd(s.q, s.k, s.v, y, lse, s.dy, ptr)
        torch.cuda.synchronize()


@pytest.mark.parametrize("lead", [1, 700])
def test_many_sequences_behind_rows_of_none(lib, lead):
    check(lib, Packed([1 + (i * 29) % 40 for i in range(130)], 2, 1, 64, BF16, seed=16, lead=lead, tail=3), "many")


@pytest.mark.parametrize("Hk", [1, 3])
def test_no_heads(lib, Hk):
    """Source heads without query heads get gradients of 0; no rows and no sequences give empty results and zeros."""
    s = Packed([40, 60], Hk, Hk, 64, F16, seed=17)
    none = s.q[:0]
    y, lse = lib.tiga_mp_attention_packed_fwd(none, s.k, s.v, s.ptr_t, want_lse=True)
    g = lib.tiga_mp_attention_packed_bwd(none, s.k, s.v, y, lse, s.dy[:0], s.ptr_t)
    torch.cuda.synchronize()
    assert y.shape == (0, 100, 64) and g["dq"].shape == (0, 100, 64)
    assert (g["dk"] == 0).all() and (g["dv"] == 0).all()
    empty = [t[:, :0] for t in (s.q, s.k, s.v)]
    y, lse = lib.tiga_mp_attention_packed_fwd(*empty, s.ptr_t[:1] * 0, want_lse=True)
    g = lib.tiga_mp_attention_packed_bwd(*empty, y, lse, empty[0], s.ptr_t[:1] * 0)
    torch.cuda.synchronize()
    assert y.shape == (Hk, 0, 64) and g["dk"].shape == (Hk, 0, 64)
    y, lse = lib.tiga_mp_attention_packed_fwd(s.q, s.k, s.v, s.ptr_t[:1], want_lse=True)      # a batch of none
    g = lib.tiga_mp_attention_packed_bwd(s.q, s.k, s.v, y, lse, s.dy, s.ptr_t[:1])
    torch.cuda.synchronize()
    assert (y == 0).all() and torch.isneginf(lse).all() and all((t == 0).all() for t in g.values())


def test_two_graphs_share_a_workspace(lib):
    """Replayed in turn on one stream."""
    one, two = Packed([300, 900], 4, 2, 64, F16, seed=18), Packed([1200], 4, 2, 64, F16, seed=19)
    ref = lib.C.byref
    size = max(lib.load().tiga_mp_attention_packed_fwd_workspace(ref(lib._packed(s.q, s.k, s.v, s.ptr_t, "hnd")[0])) for s in (one, two))
    size = max(size, *(lib.load().tiga_mp_attention_packed_bwd_workspace(ref(lib._packed(s.q, s.k, s.v, s.ptr_t, "hnd")[0])) for s in (one, two)))
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")

    def call(s, ws=None):
        y, lse = lib.tiga_mp_attention_packed_fwd(s.q, s.k, s.v, s.ptr_t, want_lse=True, ws=ws)
        return y, lse, lib.tiga_mp_attention_packed_bwd(s.q, s.k, s.v, y, lse, s.dy, s.ptr_t, ws=ws)

    want = [call(s) for s in (one, two)]
    torch.cuda.synchronize()
    graphs, got = [], []
    for s in (one, two):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got.append(call(s, ws))
        graphs.append(graph)
    for i in (0, 1, 1, 0, 1):
        graphs[i].replay()
        torch.cuda.synchronize()
        for a, b in zip(got[i][:2], want[i][:2]):
            assert torch.equal(a, b)
        assert all(torch.equal(got[i][2][n], want[i][2][n]) for n in want[i][2])


def test_given_workspaces_are_checked(lib):
    s = Packed([30], 2, 1, 64, F16, seed=20)
    for bad, err in ((torch.empty(16, dtype=torch.uint8, device="cuda"), lib.TigaError), (torch.empty(1 << 20), TypeError),
                     (torch.empty(1 << 20, 2, dtype=torch.uint8, device="cuda")[:, 0], ValueError)):
        with pytest.raises(err):
            lib.tiga_mp_attention_packed_fwd(s.q, s.k, s.v, s.ptr_t, ws=bad)


# enough tiles of long sequences that they are worked on in a planned order, cut into parts or not
PLANNED = [
    ([2300], 16, 2, 128, BF16, 0, 0),
    ([2100], 16, 16, 128, F16, 13, 150),
    ([1400, 1, 700, 0, 900], 16, 4, 128, BF16, 1, 2),
    ([600] * 4, 32, 4, 64, F16, 0, 0),
    ([520], 1, 1, 64, BF16, 0, 0),
    ([130, 4000], 6, 3, 64, F16, 5, 0),
    ([2200], 18, 3, 128, BF16, 0, 7),
]


@pytest.mark.parametrize("lens,H,Hk,D,dt,lead,tail", PLANNED)
def test_long_sequences(lib, lens, H, Hk, D, dt, lead, tail):
    check(lib, Packed(lens, H, Hk, D, dt, seed=21, lead=lead, tail=tail), f"{(lens, H, Hk, D)}")


@pytest.mark.parametrize("bad", BAD)
def test_what_is_not_finite_in_a_long_sequence(lib, bad):
    """Rows before it are as without it, in whichever part of their keys it lies."""
    s = Packed([2300], 16, 2, 128, BF16, seed=22)
    y, lse = lib.tiga_mp_attention_packed_fwd(s.q, s.k, s.v, s.ptr_t, want_lse=True)
    for row in (0, 1027, 2298):
        for t in (s.k, s.v):
            kept = t[1, row].clone()
            t[1, row, 5] = bad
            y2, lse2 = lib.tiga_mp_attention_packed_fwd(s.q, s.k, s.v, s.ptr_t, want_lse=True)
            torch.cuda.synchronize()
            t[1, row] = kept
            assert torch.equal(y2[:8], y[:8]) and torch.equal(lse2[:8], lse[:8])        # of the other source head
            assert torch.isfinite(y2[:, :row]).all() and torch.isfinite(lse2[:, :row]).all()
            # the last rounding and the weights' may differ where a neighbour moved the point that weights are relative to
            torch.testing.assert_close(y2[:, :row].float(), y[:, :row].float(), rtol=2 ** -7, atol=2 ** -6)
            if t is s.v:
                assert not torch.isfinite(y2[8:, row:, 5]).any()


def test_pointers_that_run_backwards_in_a_long_batch(lib):
    """Nothing is promised about such a call but that it stays within the tensors and ends."""
    s = Packed([2200], 16, 2, 128, F16, seed=23)
    for p in ([2200, 0], [0, 2200, 0, 2200], [1 << 30, -1, 1 << 30, 3], [-5, 1 << 30], [2200, 100, 2200, 0, 2200]):
        ptr = torch.tensor(p, dtype=torch.int32, device="cuda")
        lib.tiga_mp_attention_packed_fwd(s.q, s.k, s.v, ptr, want_lse=True)
        torch.cuda.synchronize()


@pytest.mark.parametrize("lens,H,Hk,D,dt,lead,tail", PLANNED + [
    ([], 2, 1, 64, F16, 100, 0),          # a batch of none
    ([], 3, 3, 128, BF16, 700, 0),
    ([0] * 5, 2, 2, 128, F16, 5, 600),
    ([511], 4, 1, 128, BF16, 0, 0),
    ([17], 1, 1, 64, F16, 0, 0),
    ([300] * 65, 2, 1, 128, F16, 0, 0),
])
def test_nothing_is_written_behind_a_workspace(lib, lens, H, Hk, D, dt, lead, tail):
    s = Packed(lens, H, Hk, D, dt, seed=24, lead=lead, tail=tail)
    ref = lib.C.byref(lib._packed(s.q, s.k, s.v, s.ptr_t, "hnd")[0])
    y, lse = lib.tiga_mp_attention_packed_fwd(s.q, s.k, s.v, s.ptr_t, want_lse=True)
    want = y, lse, *lib.tiga_mp_attention_packed_bwd(s.q, s.k, s.v, y, lse, s.dy, s.ptr_t).values()
    sizes = [getattr(lib.load(), f"tiga_mp_attention_packed_{n}_workspace")(ref) for n in ("fwd", "bwd")]
    whole = [torch.full((n + (1 << 20),), 0xa5, dtype=torch.uint8, device="cuda") for n in sizes]
    y, lse = lib.tiga_mp_attention_packed_fwd(s.q, s.k, s.v, s.ptr_t, want_lse=True, ws=whole[0][:sizes[0]])
    got = y, lse, *lib.tiga_mp_attention_packed_bwd(s.q, s.k, s.v, y, lse, s.dy, s.ptr_t, ws=whole[1][:sizes[1]]).values()
    torch.cuda.synchronize()
    for t, n in zip(whole, sizes):
        assert (t[n:] == 0xa5).all()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
