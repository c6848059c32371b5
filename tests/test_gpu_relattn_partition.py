"""The ways in which attention over rectangular relations cuts its work, each at a shape that takes it: items whole or
cut along the keys, narrow and wide tiles, more sequences than a wavefront has lanes, more parts than it has lanes,
heads that are no multiple of 8.  Bounds as in relattn_ref."""
import pytest
import torch

from tests import relattn_ref as R
from tests.paged_ref import Batch
from tests.test_gpu_cross_attention import both, compare as compare_cross, make
from tests.test_gpu_paged_attention import compare as compare_paged

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


@pytest.mark.parametrize("D,S,dt", [(128, 66_001, BF16), (64, 140_003, F16)])
def test_one_row_over_more_parts_than_lanes(lib, D, S, dt):
    """One item cut into a part for every resident block: the merge takes them in several turns."""
    q, k, v, _ = make(1, 2, 1, 1, S, D, dt, seed=40)
    y, lse = lib.tiga_mp_attention_cross_fwd(q, k, v, want_lse=True)
    ref, bound = R.cross(q, k, v, None, D ** -0.5)
    R.assert_within(y, ref["y"], bound["y"], "y")
    R.assert_within(lse, ref["lse"], bound["lse"], "lse")
    compare_paged(lib, Batch([(S, 1)], 1, D, 16, dt, seed=41), 2)


@pytest.mark.parametrize("dt", [F16, BF16])
def test_wide_rows_over_more_parts_than_lanes(lib, dt):
    """40 rows of one head over 33,000 keys: a wide tile cut into chunks of the least size, over 64 of them."""
    q, k, v, _ = make(1, 1, 1, 40, 33_000, 128, dt, seed=42)
    y, lse = lib.tiga_mp_attention_cross_fwd(q, k, v, want_lse=True)
    ref, bound = R.cross(q, k, v, None, 128 ** -0.5)
    R.assert_within(y, ref["y"], bound["y"], "y")
    R.assert_within(lse, ref["lse"], bound["lse"], "lse")


@pytest.mark.parametrize("H,Hk", [(5, 5), (9, 3), (16, 16), (11, 11)])
@pytest.mark.parametrize("dt", [F16, BF16])
def test_whole_items(lib, H, Hk, dt):
    """More items than run at once, of sequences of unequal lengths (one empty) and heads that fill no eight."""
    B = 2 + 1600 // (8 * H)
    q, k, v, dy = make(B, H, Hk, 130, 70, 64, dt, seed=43)
    lens = torch.tensor([(37 * b) % 71 for b in range(B)], dtype=torch.int32, device="cuda")
    got = both(lib, q, k, v, dy, lens)
    for b in (0, 1, B // 2, B - 1):
        one = slice(b, b + 1)
        ref, bound = R.cross(q[one], k[one], v[one], lens[one], 0.125, dy[one])
        for name in ref:
            R.assert_within(got[name][one], ref[name], bound[name], f"{name} of {b}")


def test_cut_items_of_unequal_sequences(lib):
    """A few wide items of lengths from 0 to 3000, cut into chunks of one size."""
    lens = torch.tensor([3000, 0, 17, 1501, 2048, 64], dtype=torch.int32, device="cuda")
    q, k, v, dy = make(6, 2, 1, 90, 3000, 128, BF16, seed=44)
    compare_cross(lib, q, k, v, dy, lens, what="cut")


@pytest.mark.parametrize("lens,H,Hk,D,page", [
    ([(300 + 7 * b, 40) for b in range(100)], 2, 1, 64, 16),                    # more sequences than lanes, wide
    ([(5 + 3 * b, 1 if b % 3 else 0) for b in range(200)], 8, 2, 128, 8),       # narrow, some without new tokens
    ([(2500, 700), (2000, 1), (1, 1), (640, 640), (0, 0), (2400, 33)], 4, 2, 128, 32),
    ([(1500, 1500)], 1, 1, 64, 64), ([(900, 900)] * 7, 12, 6, 64, 16),           # causal whole items
    ([(4000, 250)], 16, 1, 128, 16), ([(777, 300)], 3, 1, 128, 2)])              # many rows in small pages
def test_paged_partitions(lib, lens, H, Hk, D, page):
    bt = Batch(lens, Hk, D, page, BF16 if H % 2 else F16, seed=45)
    bt.spoil_unused()
    compare_paged(lib, bt, H, f"{len(lens)} sequences")


def test_repeated_calls_are_bit_identical(lib):
    for lens, H, Hk in (([(2500, 700), (2000, 1), (640, 640)], 4, 2), ([(70_000, 1), (5, 1)], 2, 1), ([(900, 900)] * 7, 12, 6)):
        bt = Batch(lens, Hk, 64, 16, F16, seed=46)
        q = bt.tokens(H)
        a = lib.tiga_mp_attention_paged_fwd(bt.cache(lib), q, bt.dst_ptr)
        b = lib.tiga_mp_attention_paged_fwd(bt.cache(lib), q, bt.dst_ptr)
        assert torch.equal(a, b)


def test_gradients_of_gradients_are_refused(lib):
    q, k, v, dy = make(1, 1, 1, 4, 5, 64, F16)
    q.requires_grad_(True)
    (g,) = torch.autograd.grad(lib.cross_attention(q, k, v), (q,), dy, create_graph=True)
    with pytest.raises(RuntimeError):
        g.sum().backward()


def test_another_device_is_refused(lib, monkeypatch):
    q, k, v, _ = make(1, 1, 1, 4, 5, 64, F16)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    with pytest.raises(ValueError):
        lib.tiga_mp_attention_cross_fwd(q, k, v)
    with pytest.raises(ValueError):
        lib.tiga_mp_rotary_fwd(q, None, lib.Rotary(lib.tiga_rotary_frequencies(64).cuda()))


def test_captured_training_step(lib):
    """Rotation, cross attention and torch.autograd.grad in one graph, replayed with eager steps of the same leaves
    alive in between."""
    q, k, v, dy = make(2, 4, 2, 60, 90, 64, BF16, seed=47)
    leaves = [t.requires_grad_(True) for t in (q, k, v)]
    rot = lib.Rotary(lib.tiga_rotary_frequencies(64).cuda())

    def step():
        y = lib.cross_attention(lib.rotary(q, None, rot), k, v)
        return (y,) + torch.autograd.grad(y, leaves, dy)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    g = torch.Generator().manual_seed(1)
    for _ in range(4):
        with torch.no_grad():
            for t in leaves:
                t.copy_(torch.randn(t.shape, generator=g).to(BF16))
        graph.replay()
        ref = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, ref))


@pytest.mark.parametrize("lens", [[(700, 1), (33, 1)], [(900, 300), (40, 2)], [(2500, 900)] * 9])
def test_output_in_the_place_of_the_queries(lib, lens):
    bt = Batch(lens, 2, 64, 16, F16, seed=48)
    q = bt.tokens(8)
    ref = lib.tiga_mp_attention_paged_fwd(bt.cache(lib), q, bt.dst_ptr)
    assert lib.tiga_mp_attention_paged_fwd(bt.cache(lib), q, bt.dst_ptr, y=q) is q
    torch.cuda.synchronize()
    assert torch.equal(q, ref)


def test_kernel_events(lib):
    """An armed pair of events is recorded around one kernel of every entry point, and by that call alone."""
    q, k, v, dy = make(2, 4, 2, 100, 300, 64, F16, seed=49)
    y, lse = lib.tiga_mp_attention_cross_fwd(q, k, v, want_lse=True)
    bt = Batch([(300, 1), (90, 5)], 2, 64, 16, F16, seed=50)
    rot = lib.Rotary(lib.tiga_rotary_frequencies(64).cuda())
    few = make(1, 2, 2, 50, 20, 64, F16, seed=51)
    fy, fl = lib.tiga_mp_attention_cross_fwd(*few[:3], want_lse=True)
    calls = [lambda: lib.tiga_mp_attention_cross_fwd(q, k, v), lambda: lib.tiga_mp_attention_cross_bwd(q, k, v, y, lse, dy),
             lambda: lib.tiga_mp_attention_cross_bwd(q, k, v, y, lse, dy, want=("dq",)),
             lambda: lib.tiga_mp_attention_cross_bwd(*few[:3], fy, fl, few[3], want=("dq",)),
             lambda: lib.tiga_mp_attention_paged_fwd(bt.cache(lib), bt.tokens(4), bt.dst_ptr),
             lambda: lib.tiga_mp_rotary_fwd(q, None, rot), lambda: lib.tiga_mp_rotary_bwd(q, None, rot),
             lambda: lib.tiga_mp_cache_append(bt.cache(lib), bt.tokens(2), bt.tokens(2), bt.dst_ptr, rot)]
    for call in calls:
        start, stop = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        start.record()
        stop.record()
        torch.cuda.synchronize()
        before = start.elapsed_time(stop)
        lib.tiga_mp_set_kernel_events(start, stop)
        call()
        torch.cuda.synchronize()
        took = start.elapsed_time(stop)
        assert took > 0 and took != before
        call()
        torch.cuda.synchronize()
        assert start.elapsed_time(stop) == took


@pytest.mark.parametrize("dt", [F16, BF16])
@pytest.mark.parametrize("D,S", [(64, 3), (64, 127), (64, 128), (64, 129), (128, 2), (128, 63), (128, 64), (128, 65)])
def test_gradients_around_one_tile_of_sources(lib, D, S, dt):
    """Up to one tile of sources delta comes with dq, from them; unequal lengths, padding never seen, any choice of gradients."""
    q, k, v, dy = make(4, 6, 2, 75, S, D, dt, seed=60 + S)
    lens = torch.tensor([S, 0, 1, S - 1], dtype=torch.int32, device="cuda")
    kc, vc = k.clone(), v.clone()
    for b, n in enumerate(lens.tolist()):
        kc[b, :, n:], vc[b, :, n:] = 0, 0
        k[b, :, n:], v[b, :, n:] = float("nan"), float("inf")
    got = both(lib, q, k, v, dy, lens)
    ref, bound = R.cross(q, kc, vc, lens, D ** -0.5, dy)
    for name in ("lse", "y", "dv", "dq", "dk"):
        R.assert_within(got[name], ref[name], bound[name], name)
    for want in (("dq",), ("dk",), ("dv",), ("dq", "dv")):
        some = lib.tiga_mp_attention_cross_bwd(q, k, v, got["y"], got["lse"], dy, lens, want=want)
        assert list(some) == list(want) and all(torch.equal(some[n], got[n]) for n in want)
