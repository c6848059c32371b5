"""Attention of new tokens over a paged cache against 64 bits on the CPU; the bounds are derived in relattn_ref."""
import pytest
import torch

from tests import relattn_ref as R
from tests.paged_ref import Batch

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


def reference(bt, q, scale):
    """q [heads, num_dst, width].  Outputs and bounds; rows of no sequence stay NaN."""
    H, N, D = q.shape
    y = torch.full((H, N, D), float("nan"), dtype=torch.float64)
    lse = torch.full((H, N), float("nan"), dtype=torch.float64)
    by, bl = torch.zeros_like(y), torch.zeros_like(lse)
    qd = q.double().cpu()
    for b, (n, c) in enumerate(bt.lens):
        if c == 0:
            continue
        k, v = (t.double() for t in bt.gathered(b))
        m = k.shape[1]
        seen = torch.arange(m)[None, :] <= (n - c + torch.arange(c))[:, None]
        rows = slice(bt.ptr[b], bt.ptr[b] + c)
        for h in range(H):
            j = h // (H // bt.kv_heads)
            f = R.rows(qd[h, rows], k[j], v[j], seen, scale)
            y[h, rows], lse[h, rows] = f["y"], f["lse"]
            by[h, rows], bl[h, rows] = f["y_bound"](bt.dt), f["lse_bound"]
    return y, lse, by, bl


def compare(lib, bt, heads, what="", layout="hnd", scale=None):
    q = bt.tokens(heads, layout == "nhd")
    y, lse = lib.tiga_mp_attention_paged_fwd(bt.cache(lib), q, bt.dst_ptr, scale, want_lse=True, layout=layout)
    torch.cuda.synchronize()
    if layout == "nhd":
        q, y = q.permute(1, 0, 2), y.permute(1, 0, 2)
    ry, rl, by, bl = reference(bt, q, bt.width ** -0.5 if scale is None else scale)
    n = bt.rows
    R.assert_within(lse[:, :n], rl[:, :n], bl[:, :n], what + " lse")
    R.assert_within(y[:, :n], ry[:, :n], by[:, :n], what + " y")


# lengths (with the new tokens, new tokens), heads, source heads, width, page, type
CASES = [
    ([(1, 1)], 1, 1, 64, 16, F16),
    ([(5, 1), (17, 1), (16, 1), (33, 1)], 4, 2, 128, 16, BF16),
    ([(1000, 1)], 8, 1, 128, 32, F16),
    ([(4001, 1), (1, 1), (63, 1), (65, 1), (700, 1)], 8, 2, 64, 64, BF16),
    ([(40, 40)], 2, 2, 64, 16, F16),
    ([(129, 129), (300, 7), (64, 64), (10, 1)], 4, 1, 128, 16, BF16),
    ([(2000, 500), (37, 1)], 3, 3, 128, 128, F16),
    ([(100, 0), (50, 3), (0, 0), (9, 9)], 6, 2, 64, 8, BF16),
    ([(31, 5)], 32, 1, 128, 1, F16),
    ([(777, 130)], 5, 1, 64, 1024, BF16),
    ([(3000, 2), (2999, 17), (100, 16), (100, 33)], 4, 4, 64, 32, F16),
    ([(20 + 13 * i, 1 + i % 2) for i in range(70)], 2, 1, 64, 16, BF16),
    ([(257, 1)] * 3, 12, 12, 128, 256, BF16),
    ([(6000, 1), (12, 1)], 40, 2, 128, 16, F16),
    ([(512, 512), (511, 511)], 2, 1, 128, 64, F16),
]


@pytest.mark.parametrize("lens,H,Hk,D,page,dt", CASES)
def test_against_64_bits(lib, lens, H, Hk, D, page, dt):
    bt = Batch(lens, Hk, D, page, dt, seed=len(lens) + page)
    bt.spoil_unused()
    lib.tiga_cache_validate(bt.cache(lib), bt.num_dst, bt.dst_ptr)
    compare(lib, bt, H, f"{(len(lens), lens[0], H, Hk, D, page)}")


@pytest.mark.parametrize("lens", [[(300, 1), (40, 1)], [(300, 100), (40, 1)]])
def test_pages_stored_rows_first(lib, lens):
    bt = Batch(lens, 2, 64, 16, BF16, seed=3, rows_first=True)
    compare(lib, bt, 4, layout="nhd", scale=0.2)


@pytest.mark.parametrize("lens", [[(300, 1), (40, 1)], [(300, 100), (40, 2)]])
def test_rows_behind_the_last_sequence_stay(lib, lens):
    bt = Batch(lens, 2, 64, 16, F16, seed=4, tail=5)
    q = bt.tokens(4)
    y = torch.full_like(q, 3.0)
    out = lib.tiga_mp_attention_paged_fwd(bt.cache(lib), q, bt.dst_ptr, y=y)
    torch.cuda.synchronize()
    assert out is y and (y[:, bt.rows:] == 3.0).all() and not (y[:, :bt.rows] == 3.0).all(2).any()


@pytest.mark.parametrize("new", [1, 40])
def test_bad_pages_give_nan_where_they_are_needed(lib, new):
    """A page outside the cache, and a length past the table: rows that need them are NaN, all others right."""
    bt = Batch([(300, new), (200, new), (120, new)], 2, 128, 16, F16, seed=5)
    q = bt.tokens(4)
    good = lib.tiga_mp_attention_paged_fwd(bt.cache(lib), q, bt.dst_ptr)
    for bad in (-1, bt.num_pages, 2 ** 31 - 1, -2 ** 31):
        table, length = bt.table.clone(), bt.length.clone()
        table[0, 5] = bad
        length[2] = bt.table.shape[1] * 16 + 77
        cache = lib.KvCache(bt.k, bt.v, table, length)
        y, lse = lib.tiga_mp_attention_paged_fwd(cache, q, bt.dst_ptr, want_lse=True)
        torch.cuda.synchronize()
        p = bt.ptr
        assert torch.isnan(y[:, p[0]:p[1]]).all() and torch.isnan(lse[:, p[0]:p[1]]).all()
        assert torch.equal(y[:, p[1]:p[2]], good[:, p[1]:p[2]])
        assert torch.isnan(y[:, p[2]:p[3]]).all()
        for n, code in ((bt.num_dst, lib.TIGA_EGRAPH),):
            with pytest.raises(lib.TigaError) as e:
                lib.tiga_cache_validate(cache, n, bt.dst_ptr)
            assert e.value.code == code


def test_a_bad_page_within_the_new_tokens(lib):
    """Rows before the bad page's first position do not need it."""
    bt = Batch([(200, 100)], 1, 64, 16, BF16, seed=6)
    q = bt.tokens(2)
    good = lib.tiga_mp_attention_paged_fwd(bt.cache(lib), q, bt.dst_ptr)
    bt.table[0, 8] = -1                      # positions 128 to 143; the new tokens are 100 to 199
    y = lib.tiga_mp_attention_paged_fwd(bt.cache(lib), q, bt.dst_ptr)
    torch.cuda.synchronize()
    assert torch.equal(y[:, :28], good[:, :28]) and torch.isnan(y[:, 28:]).all()


def test_more_new_tokens_than_positions(lib):
    """Rows without a position have nothing to read: y = 0, lse = -inf."""
    bt = Batch([(10, 10)], 1, 64, 16, F16, seed=7)
    q = bt.tokens(2)
    bt.length[0] = 4
    y, lse = lib.tiga_mp_attention_paged_fwd(bt.cache(lib), q, bt.dst_ptr, want_lse=True)
    torch.cuda.synchronize()
    assert (y[:, :6] == 0).all() and torch.isneginf(lse[:, :6]).all() and torch.isfinite(lse[:, 6:]).all()
    k, v = (t[0, :4].double() for t in bt.gathered(0))
    for h in range(2):
        f = R.rows(q[h, 6:].double().cpu(), k, v, torch.ones(4, 4).tril().bool(), 64 ** -0.5)
        R.assert_within(y[h, 6:], f["y"], f["y_bound"](F16), "rows with positions")


def test_pointers_that_run_backwards_stay_inside(lib):
    """Nothing is promised about such a call but that it stays within the tensors and ends."""
    bt = Batch([(50, 5), (60, 6), (70, 7)], 1, 64, 16, F16, seed=8)
    q = bt.tokens(2)
    for ptr in ([0, 11, 5, 18], [-7, 5, 11, 18], [0, 5, 11, 10_000], [18, 5, 0, -1], [9, 9, 9, 9]):
        dst_ptr = torch.tensor(ptr, dtype=torch.int32, device="cuda")
        y = lib.tiga_mp_attention_paged_fwd(bt.cache(lib), q, dst_ptr)
        torch.cuda.synchronize()
        assert y.shape == q.shape


def test_shared_pages(lib):
    """Two sequences that share their first pages (a forked prompt) read the same keys."""
    bt = Batch([(100, 1), (100, 1)], 2, 64, 16, BF16, seed=9)
    bt.table[1] = bt.table[0]
    q = bt.tokens(2)
    q[:, 1] = q[:, 0]
    y = lib.tiga_mp_attention_paged_fwd(bt.cache(lib), q, bt.dst_ptr)
    assert torch.equal(y[:, 0], y[:, 1])


@pytest.mark.parametrize("lens", [[(5000, 1), (3, 1)], [(900, 300), (80, 1), (700, 2)]])
def test_repeated_and_in_two_streams(lib, lens):
    a, b = Batch(lens, 2, 128, 16, BF16, seed=10), Batch(lens[::-1], 1, 64, 32, F16, seed=11)
    qa, qb = a.tokens(8), b.tokens(8)
    ra = lib.tiga_mp_attention_paged_fwd(a.cache(lib), qa, a.dst_ptr)
    rb = lib.tiga_mp_attention_paged_fwd(b.cache(lib), qb, b.dst_ptr)
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(s1):
            ya = lib.tiga_mp_attention_paged_fwd(a.cache(lib), qa, a.dst_ptr)
        with torch.cuda.stream(s2):
            yb = lib.tiga_mp_attention_paged_fwd(b.cache(lib), qb, b.dst_ptr)
        torch.cuda.synchronize()
        assert torch.equal(ya, ra) and torch.equal(yb, rb)


def test_offsets_past_32_bits(lib):
    """A cache of over 4 GiB (and over 2^31 elements) a side whose last pages are used."""
    page, Hk, D = 64, 2, 128
    pages = (1 << 31) // (page * Hk * D) + 40
    k = torch.zeros(pages, Hk, page, D, dtype=BF16, device="cuda")
    v = torch.zeros(pages, Hk, page, D, dtype=BF16, device="cuda")
    bt = Batch([(300, 1), (200, 70)], Hk, D, page, BF16, seed=12)
    used = torch.arange(pages - bt.num_pages, pages, device="cuda")
    k[used], v[used] = bt.k, bt.v
    table = torch.where(bt.table >= 0, bt.table + (pages - bt.num_pages), bt.table).to(torch.int32)
    q = bt.tokens(4)
    small = lib.tiga_mp_attention_paged_fwd(bt.cache(lib), q, bt.dst_ptr)
    y = lib.tiga_mp_attention_paged_fwd(lib.KvCache(k, v, table, bt.length), q, bt.dst_ptr)
    assert torch.equal(y, small)


def test_captured_and_replayed(lib):
    """A generation step in a graph: lengths, tables and tokens change between the replays."""
    bt = Batch([(700, 1), (600, 1), (90, 1)], 2, 128, 16, F16, seed=13)
    cache = bt.cache(lib)
    q = bt.tokens(8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        lib.tiga_mp_attention_paged_fwd(cache, q, bt.dst_ptr)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, lse = lib.tiga_mp_attention_paged_fwd(cache, q, bt.dst_ptr, want_lse=True)
    for i in range(4):
        q.copy_(bt.tokens(8))
        bt.length.copy_(torch.tensor([[700, 1, 16], [17, 600, 90], [1, 2, 3], [699, 599, 0]][i], dtype=torch.int32))
        graph.replay()
        ref, rl = lib.tiga_mp_attention_paged_fwd(cache, q, bt.dst_ptr, want_lse=True)
        torch.cuda.synchronize()
        assert torch.equal(y, ref) and torch.equal(lse, rl), i


def test_empty_calls(lib):
    bt = Batch([(40, 4)], 2, 64, 16, F16)
    y = lib.tiga_mp_attention_paged_fwd(bt.cache(lib), bt.tokens(4)[:, :0], torch.zeros(2, dtype=torch.int32, device="cuda"))
    assert y.shape == (4, 0, 64)
    none = lib.KvCache(bt.k, bt.v, bt.table[:0], bt.length[:0])
    q = bt.tokens(4)
    y = torch.full_like(q, 2.0)
    lib.tiga_mp_attention_paged_fwd(none, q, torch.zeros(1, dtype=torch.int32, device="cuda"), y=y)
    assert (y == 2.0).all()


@pytest.mark.parametrize("new", [1, 40])
def test_batch_strides_of_packed_rows_are_not_used(lib, new):
    """Whatever a C caller leaves in the batch strides of q and y (one packed axis has none)."""
    import ctypes as C
    bt = Batch([(100, new), (60, new), (300, new)], 2, 64, 16, F16, seed=14)
    q = bt.tokens(4)
    ref = lib.tiga_mp_attention_paged_fwd(bt.cache(lib), q, bt.dst_ptr)
    y = torch.zeros_like(q)
    L, cache = lib.load(), bt.cache(lib)
    _, qv = lib._rows(q, "q", lib._AXES["hnd"])
    _, yv = lib._rows(y, "y", lib._AXES["hnd"])
    qv.batch = yv.batch = 8
    ws = lib._workspace(L.tiga_mp_attention_paged_fwd_workspace(cache.ref, bt.num_dst, 4), q.device)
    assert L.tiga_mp_attention_paged_fwd(cache.ref, bt.num_dst, lib._ptr(bt.dst_ptr), 4, C.byref(qv), 0.125, C.byref(yv), None,
                                         lib._ptr(ws), ws.numel(), lib._stream()) == lib.TIGA_OK
    torch.cuda.synchronize()
    assert torch.equal(y, ref)


def test_a_workspace_of_a_larger_problem(lib):
    """One workspace, sized for the largest, serves smaller problems of either tile shape, filled with anything before."""
    big = Batch([(3000, 200)] * 4, 2, 128, 16, BF16, seed=15)
    L = lib.load()
    ws = lib._workspace(L.tiga_mp_attention_paged_fwd_workspace(big.cache(lib).ref, big.num_dst, 8), torch.device("cuda"))
    for lens in ([(3000, 200)] * 4, [(2000, 1)] * 4, [(700, 90)], [(5, 1), (2900, 3)]):
        bt = Batch(lens, 2, 128, 16, BF16, seed=16)
        q = bt.tokens(8)
        ws.fill_(0xFF)
        y = lib.tiga_mp_attention_paged_fwd(bt.cache(lib), q, bt.dst_ptr, ws=ws)
        assert torch.equal(y, lib.tiga_mp_attention_paged_fwd(bt.cache(lib), q, bt.dst_ptr))
