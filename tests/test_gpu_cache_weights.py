"""Accumulated attention weights of cached positions against 64 bits on the CPU.

A weight exp(s - lse) is off by what its score is (relattn_ref: es), and by the rounding of lse * log2 e and of the exponent's
argument, 2^-22 (|lse| + 1) together; a sum over n rows by R.sums(n) of the sum; decay * old and its addition by 2^-22 of
them."""
import pytest
import torch

from tests import relattn_ref as R
from tests.paged_ref import Batch

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


def reference(bt, q, lse, weights, decay, scale):
    """out and its bound; NaN where no position has a cell."""
    P, Hk, page = weights.shape
    out = torch.full(weights.shape, float("nan"), dtype=torch.float64)
    bound = torch.zeros_like(out)
    qd, ld, wd = q.double().cpu(), lse.double().cpu(), weights.double().cpu()
    H, D = q.shape[0], q.shape[2]
    table = bt.table.cpu()
    for b, (n, c) in enumerate(bt.lens):
        if n <= 0:
            continue
        k, _ = (t.double() for t in bt.gathered(b))
        at = torch.arange(n)
        ids, slot = table[b].long()[at // page], at % page
        seen = at[None, :] <= (n - c + torch.arange(c))[:, None]
        rows = slice(bt.ptr[b], bt.ptr[b] + c)
        for j in range(Hk):
            new, err = torch.zeros(n, dtype=torch.float64), torch.zeros(n, dtype=torch.float64)
            for h in range(j * (H // Hk), (j + 1) * (H // Hk)):
                s = qd[h, rows] @ k[j].t() * scale
                es = 2 * (D + 8) * 2.0 ** -24 * scale * (qd[h, rows].abs() @ k[j].abs().t()) + 2.0 ** -22 * s.abs() + 2.0 ** -21
                l = ld[h, rows][:, None]
                p = torch.where(seen & (l > -torch.inf), torch.exp(s - l), 0.0)
                new += p.sum(0)
                err += torch.where(p > 0, p * (es + 2.0 ** -22 * (l.abs() + 1)), 0.0).sum(0)
            old = torch.where(at < n - c, decay * wd[ids, j, slot], 0.0)
            out[ids, j, slot] = new + old
            bound[ids, j, slot] = 2 * err + R.sums(c * (H // Hk)) * new + 2.0 ** -22 * (new + old.abs()) + 2.0 ** -126
    return out, bound


def compare(lib, bt, H, what, decay=1.0, scale=None, layout="hnd", in_place=False):
    q = bt.tokens(H, layout == "nhd")
    cache = bt.cache(lib)
    _, lse = lib.tiga_mp_attention_paged_fwd(cache, q, bt.dst_ptr, scale, want_lse=True, layout=layout)
    g = torch.Generator().manual_seed(99)
    weights = torch.rand(bt.num_pages, bt.kv_heads, bt.page, generator=g).cuda() * 3
    given = weights.clone()
    out = weights if in_place else torch.full_like(weights, -7.0)
    got = lib.tiga_mp_cache_weights(cache, q, lse, bt.dst_ptr, weights, None if in_place else out, decay, scale, layout)
    torch.cuda.synchronize()
    assert got is out
    qh = q.permute(1, 0, 2) if layout == "nhd" else q
    ref, bound = reference(bt, qh, lse, given, decay, bt.width ** -0.5 if scale is None else scale)
    cells = ~torch.isnan(ref)
    R.assert_within(got.cpu()[cells], ref[cells], bound[cells], what)
    rest = got.cpu()[~cells]
    assert torch.equal(rest, given.cpu()[~cells] if in_place else torch.full_like(rest, -7.0)), "cells of no position"
    if not in_place:
        assert torch.equal(weights, given)
    return got


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
    ([(20 + 13 * i, 1 + i % 2) for i in range(70)], 2, 1, 64, 16, BF16),
    ([(257, 1)] * 3, 12, 12, 128, 256, BF16),
    ([(1500, 900), (300, 300)], 2, 1, 128, 2, BF16),
    ([(700, 257), (128, 128), (64, 17)], 16, 2, 64, 32, F16),
    # long chunks over few keys, whose rows are cut; beside next tokens
    ([(2100, 2000), (900, 1), (70, 5), (1300, 1200)], 8, 1, 128, 16, BF16),
    ([(3000, 2900)], 4, 1, 64, 64, F16),
    ([(130 + i, 20 + i) for i in range(70)], 2, 1, 64, 16, BF16),
]


@pytest.mark.parametrize("lens,H,Hk,D,page,dt", CASES)
def test_against_64_bits(lib, lens, H, Hk, D, page, dt):
    bt = Batch(lens, Hk, D, page, dt, seed=len(lens) + page)
    bt.spoil_unused()
    compare(lib, bt, H, f"{(len(lens), lens[0], H, Hk, D, page)}")


@pytest.mark.parametrize("lens", [[(300, 1), (40, 1)], [(300, 100), (40, 2)], [(400, 333), (40, 1)]])
@pytest.mark.parametrize("decay", [0.0, 0.5, 1.0])
def test_in_place_and_layouts(lib, lens, decay):
    compare(lib, Batch(lens, 2, 64, 16, F16, seed=3, tail=5), 4, "in place", decay=decay, in_place=True)
    compare(lib, Batch(lens, 2, 128, 16, BF16, seed=4, rows_first=True), 4, "rows first", decay=decay, scale=0.2, layout="nhd")


@pytest.mark.parametrize("new", [1, 40, 300])
def test_old_weights_of_new_positions_do_not_count(lib, new):
    """What lies in the cells of the new tokens, NaN among it, is overwritten."""
    bt = Batch([(600, new)], 1, 64, 16, F16, seed=5)
    q = bt.tokens(2)
    cache = bt.cache(lib)
    _, lse = lib.tiga_mp_attention_paged_fwd(cache, q, bt.dst_ptr, want_lse=True)
    a = torch.zeros(bt.num_pages, 1, 16, device="cuda")
    want = lib.tiga_mp_cache_weights(cache, q, lse, bt.dst_ptr, a, torch.zeros_like(a))
    for p in range(600 - new, 600):
        a[int(bt.table[0, p // 16]), 0, p % 16] = float("nan")
    got = lib.tiga_mp_cache_weights(cache, q, lse, bt.dst_ptr, a, torch.zeros_like(a))
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.isfinite(got).all()


@pytest.mark.parametrize("new", [1, 300])
def test_what_is_not_finite(lib, new):
    """A key that is NaN has a weight of NaN, the others theirs; a query that is NaN reaches what it sees."""
    bt = Batch([(900, new)], 1, 64, 16, BF16, seed=6)
    q = bt.tokens(2)
    cache = bt.cache(lib)
    _, lse = lib.tiga_mp_attention_paged_fwd(cache, q, bt.dst_ptr, want_lse=True)
    w = torch.rand(bt.num_pages, 1, 16, device="cuda")
    good = lib.tiga_mp_cache_weights(cache, q, lse, bt.dst_ptr, w, torch.zeros_like(w))
    cell = lambda p: (int(bt.table[0, p // 16]), 0, p % 16)
    page, _, row = cell(444)
    kept = bt.k[page, 0, row].clone()
    bt.k[page, 0, row, 3] = float("nan")
    got = lib.tiga_mp_cache_weights(cache, q, lse, bt.dst_ptr, w, torch.zeros_like(w))
    torch.cuda.synchronize()
    assert torch.isnan(got[cell(444)])
    got[cell(444)] = good[cell(444)]
    assert torch.equal(got, good)
    bt.k[page, 0, row] = kept
    if new > 1:
        q[1, 100] = float("nan")                     # at position 600 + 100
        got = lib.tiga_mp_cache_weights(cache, q, lse, bt.dst_ptr, w, torch.zeros_like(w))
        torch.cuda.synchronize()
        for p in (0, 444, 700):
            assert torch.isnan(got[cell(p)])
        for p in range(701, 900):
            assert got[cell(p)] == good[cell(p)]


def test_bad_pages_lengths_and_rows(lib):
    """Positions without a page have no cell; rows that saw nothing give nothing; a length past the table ends with it."""
    bt = Batch([(300, 1), (200, 1), (10, 10)], 1, 64, 16, F16, seed=7)
    q = bt.tokens(2)
    w = torch.rand(bt.num_pages, 1, 16, device="cuda")
    lse = torch.zeros(2, bt.num_dst, device="cuda")
    good = lib.tiga_mp_cache_weights(bt.cache(lib), q, lse, bt.dst_ptr, w, torch.full_like(w, -1.0))
    table, length = bt.table.clone(), bt.length.clone()
    lost = table[0, 5].clone()
    for bad in (-1, bt.num_pages, 2 ** 31 - 1, -2 ** 31):
        table[0, 5] = bad
        got = lib.tiga_mp_cache_weights(lib.KvCache(bt.k, bt.v, table, length), q, lse, bt.dst_ptr, w, torch.full_like(w, -1.0))
        torch.cuda.synchronize()
        assert (got[lost] == -1.0).all()
        got[lost] = good[lost]
        assert torch.equal(got, good), bad
    lse[:] = float("-inf")
    got = lib.tiga_mp_cache_weights(bt.cache(lib), q, lse, bt.dst_ptr, w, w.clone())
    torch.cuda.synchronize()
    old = w[int(bt.table[0, 0])]
    assert torch.equal(got[int(bt.table[0, 0])], old) and (got[int(bt.table[2, 0]), 0, :10] == 0).all()
    length[0] = 10_000
    lib.tiga_mp_cache_weights(lib.KvCache(bt.k, bt.v, bt.table, length), q, lse, bt.dst_ptr, w, w.clone())
    torch.cuda.synchronize()


def test_pointers_that_run_backwards_stay_inside(lib):
    bt = Batch([(300, 20), (200, 30)], 1, 64, 16, F16, seed=8)
    q = bt.tokens(2)
    lse, w = torch.zeros(2, bt.num_dst, device="cuda"), torch.rand(bt.num_pages, 1, 16, device="cuda")
    for p in ([50, 20, 0], [-5, 1 << 30, 3], [0, 50, 1 << 30]):
        bt.dst_ptr.copy_(torch.tensor(p, dtype=torch.int32))
        lib.tiga_mp_cache_weights(bt.cache(lib), q, lse, bt.dst_ptr, w, w.clone())
        torch.cuda.synchronize()


def test_captured(lib):
    bt = Batch([(700, 1), (650, 3), (90, 1)], 2, 128, 16, BF16, seed=11)
    q, cache = bt.tokens(8), bt.cache(lib)
    w = torch.zeros(bt.num_pages, 2, 16, device="cuda")

    def call():
        y, lse = lib.tiga_mp_attention_paged_fwd(cache, q, bt.dst_ptr, want_lse=True)
        return lib.tiga_mp_cache_weights(cache, q, lse, bt.dst_ptr, w, decay=0.5)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    w.zero_()
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    got = w.clone()
    w.zero_()
    call()
    call()
    torch.cuda.synchronize()
    assert torch.equal(got, w) and got.abs().sum() > 0
