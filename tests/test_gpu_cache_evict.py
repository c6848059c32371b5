"""Eviction from a paged cache: exactly the positions, rows and weights that the definition keeps."""
import pytest
import torch

from tests.paged_ref import Batch

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


class Case:
    def __init__(self, lens, Hk, D, page, dt, keep, recent, kind="spread", to_page=None, seed=0, rows_first=False):
        self.bt = bt = Batch([(n, 0) for n in lens], Hk, D, page, dt, seed=seed, rows_first=rows_first)
        self.to = Batch([(min(n, keep), 0) for n in lens], Hk, D, to_page or page, dt, seed=seed + 1, rows_first=rows_first)
        self.keep, self.recent, self.lens = keep, recent, lens
        g = torch.Generator().manual_seed(seed + 2)
        w = torch.randn(bt.num_pages, Hk, page, generator=g)
        if kind == "equal":
            w = torch.full_like(w, 0.25)
        elif kind == "few":                      # four values, zeros of both signs among them
            w = torch.tensor([0.0, -0.0, 1.0, 2.5])[torch.randint(0, 4, w.shape, generator=g)]
        elif kind == "wild":
            pick = torch.randint(0, 8, w.shape, generator=g)
            for i, v in enumerate((float("inf"), float("-inf"), float("nan"), 1e-42, -1e-42)):
                w[pick == i] = v
        elif kind == "near":                     # equal but for the last bits
            w = (torch.randint(0, 5, w.shape, generator=g) + 0x3f800000).to(torch.int32).view(torch.float32)
        self.weights = w.cuda()
        self.to_weights = torch.full((self.to.num_pages, Hk, self.to.page), -7.0, device="cuda")

    def expected(self):
        """kept, and the destination's pages and weights."""
        bt, to = self.bt, self.to
        k, v, w = to.k.cpu().clone(), to.v.cpu().clone(), self.to_weights.cpu().clone()
        fk, fv, fw = bt.k.cpu(), bt.v.cpu(), self.weights.cpu()
        kept = torch.full((len(self.lens), bt.kv_heads, self.keep), -1, dtype=torch.int32)
        for b, n in enumerate(self.lens):
            at = torch.arange(n)
            ids, slot = bt.table[b].long().cpu()[at // bt.page], at % bt.page
            last = min(self.recent, self.keep, n)
            for j in range(bt.kv_heads):
                x = fw[ids, j, slot].double()
                rank = torch.where(torch.isnan(x), torch.full_like(x, 1e300), x.clamp(min=-1e299, max=1e299))[: n - last]
                some = torch.sort(-rank, stable=True).indices[: min(self.keep, n) - last].sort().values
                stay = torch.cat([some, at[n - last:]])
                place = torch.arange(stay.numel())
                tid, ts = to.table[b].long().cpu()[place // to.page], place % to.page
                k[tid, j, ts], v[tid, j, ts], w[tid, j, ts] = fk[ids[stay], j, slot[stay]], fv[ids[stay], j, slot[stay]], fw[ids[stay], j, slot[stay]]
                kept[b, j, : stay.numel()] = stay.to(torch.int32)
        return kept, k, v, w


def same(a, b):
    """Equal bits (NaN too)."""
    kind = torch.int32 if a.dtype == torch.float32 else torch.int16
    return torch.equal(a.cpu().contiguous().view(kind), b.cpu().contiguous().view(kind))


CASES = [
    ([1], 1, 64, 16, F16, 1, 0, "spread"),
    ([5], 2, 64, 16, F16, 4, 0, "spread"),
    ([5], 2, 64, 16, F16, 1, 1, "spread"),
    ([100, 60, 61, 0, 1], 2, 128, 16, BF16, 60, 7, "spread"),
    ([100, 300, 256], 1, 64, 16, F16, 100, 0, "equal"),
    ([1000, 999], 3, 64, 32, BF16, 500, 500, "few"),
    ([1000, 4096, 4097, 4095], 2, 64, 64, F16, 777, 31, "few"),
    ([513, 700], 2, 128, 8, BF16, 512, 100, "wild"),
    ([5000, 9000], 1, 64, 128, F16, 3001, 64, "near"),
    ([40, 30], 4, 64, 1, F16, 20, 3, "spread"),
    ([90, 33], 1, 128, 2, BF16, 32, 5, "few"),
    ([33_000, 100], 1, 64, 64, F16, 1000, 10, "few"),
    ([70_001], 1, 64, 16, BF16, 65_000, 1, "wild"),
    ([50_000, 8192, 8193, 400, 0], 2, 64, 32, F16, 8000, 4000, "spread"),
    ([40_000, 33_000], 1, 64, 64, BF16, 500, 500, "near"),
    ([60_000], 3, 64, 16, F16, 20_000, 100, "near"),
    ([40_000, 9_000], 1, 64, 128, F16, 12_000, 7, "equal"),
    ([35_000], 1, 64, 1, F16, 30_000, 9, "wild"),
    ([34_000 - 100 * (i % 300) for i in range(300)], 1, 64, 64, F16, 900, 10, "few"),   # more lists than compute units
    ([20 + 5 * (i % 30) for i in range(70)], 3, 64, 16, F16, 90, 9, "spread"),
]


@pytest.mark.parametrize("lens,Hk,D,page,dt,keep,recent,kind", CASES)
def test_exactly(lib, lens, Hk, D, page, dt, keep, recent, kind):
    c = Case(lens, Hk, D, page, dt, keep, recent, kind, seed=len(lens) + keep)
    kept, k, v, w = c.expected()
    to = c.to.cache(lib)
    to.length.fill_(-5)
    got = lib.tiga_mp_cache_evict(c.bt.cache(lib), c.weights, to, c.to_weights, keep=keep, recent=recent)
    torch.cuda.synchronize()
    assert torch.equal(got.cpu(), kept)
    assert same(c.to.k, k) and same(c.to.v, v) and same(c.to_weights, w)
    assert to.length.tolist() == [min(n, keep) for n in lens]


@pytest.mark.parametrize("page,to_page", [(16, 64), (64, 16), (16, 1), (2, 16)])
def test_other_pages_and_rows_first(lib, page, to_page):
    c = Case([300, 100], 2, 64, page, BF16, 130, 20, "few", to_page=to_page, seed=3, rows_first=True)
    kept, k, v, w = c.expected()
    before = c.to_weights.clone()
    got = lib.tiga_mp_cache_evict(c.bt.cache(lib), c.weights, c.to.cache(lib), keep=130, recent=20)   # weights not wanted
    torch.cuda.synchronize()
    assert torch.equal(got.cpu(), kept) and same(c.to.k, k) and same(c.to.v, v) and torch.equal(before, c.to_weights)


@pytest.mark.parametrize("lens,keep,recent", [([300, 100, 0, 131], 130, 20), ([5000], 4999, 0), ([64, 64], 64, 1), ([700], 1, 0)])
@pytest.mark.parametrize("page", [1, 16, 64])
def test_in_place(lib, lens, keep, recent, page):
    """The same rows as into another cache; the rest of the pages is as it was."""
    c = Case(lens, 2, 128, page, F16, keep, recent, "few", seed=4)
    kept, k, v, w = c.expected()
    bt, cache = c.bt, c.bt.cache(lib)
    k0, v0, w0 = bt.k.clone(), bt.v.clone(), c.weights.clone()
    got = lib.tiga_mp_cache_evict(cache, c.weights, keep=keep, recent=recent)
    torch.cuda.synchronize()
    assert torch.equal(got.cpu(), kept) and cache.length.tolist() == [min(n, keep) for n in lens]
    mine = torch.zeros(bt.num_pages, page, dtype=torch.bool)
    for b, n in enumerate(lens):
        at = torch.arange(min(n, keep))
        ids, slot = bt.table[b].long().cpu()[at // page], at % page
        tid, ts = c.to.table[b].long().cpu()[at // page], at % page
        mine[ids, slot] = True
        for x, y in ((bt.k.cpu()[ids, :, slot], k[tid, :, ts]), (bt.v.cpu()[ids, :, slot], v[tid, :, ts]),
                     (c.weights.cpu()[ids, :, slot], w[tid, :, ts])):
            assert same(x, y)
    for x, y in ((bt.k, k0), (bt.v, v0), (c.weights, w0)):
        x, y = x.cpu().transpose(1, 2), y.cpu().transpose(1, 2)
        assert same(x[~mine], y[~mine])


def test_pages_of_one_pool(lib):
    """Both caches' pages lie in the same tensors, and the weights'."""
    c = Case([300, 100], 2, 64, 16, F16, 130, 20, "spread", seed=5)
    kept, k, v, w = c.expected()
    bt, to = c.bt, c.to
    pk, pv, pw = torch.cat([bt.k, to.k]), torch.cat([bt.v, to.v]), torch.cat([c.weights, c.to_weights])
    a = lib.KvCache(pk, pv, bt.table, bt.length)
    z = lib.KvCache(pk, pv, torch.where(to.table >= 0, to.table + bt.num_pages, to.table), to.length)
    got = lib.tiga_mp_cache_evict(a, pw, z, pw, keep=130, recent=20)
    torch.cuda.synchronize()
    assert torch.equal(got.cpu(), kept)
    assert same(pk, torch.cat([bt.k.cpu(), k])) and same(pv, torch.cat([bt.v.cpu(), v])) and same(pw, torch.cat([c.weights.cpu(), w]))


def test_bad_pages_and_lengths(lib):
    """A position without a page is the first to go, and nothing is stored for one; a new place without a page is left out;
    a negative length is 0, one past the table ends with it."""
    c = Case([300, 100, 50], 1, 64, 16, F16, 130, 20, "spread", seed=6)
    bt, to = c.bt, c.to
    bt.table[0, 3] = bt.num_pages
    to.table[1, 2] = -1
    bt.length[2] = -9
    z = to.cache(lib)
    kept = lib.tiga_mp_cache_evict(bt.cache(lib), c.weights, z, c.to_weights, keep=130, recent=20)
    torch.cuda.synchronize()
    assert not ((kept[0] >= 48) & (kept[0] < 64)).any() and (kept[0] >= 0).all()
    assert (kept[1, 0, :100].cpu() == torch.arange(100)).all() and (kept[1, 0, 100:] == -1).all()
    assert (kept[2] == -1).all() and z.length.tolist() == [130, 100, 0]
    bt.length[2] = 1 << 30
    kept = lib.tiga_mp_cache_evict(bt.cache(lib), c.weights, z, c.to_weights, keep=130, recent=20)
    torch.cuda.synchronize()
    assert kept.max() < bt.table.shape[1] * 16


def test_captured(lib):
    c = Case([300, 100, 200], 2, 64, 16, F16, 130, 20, "few", seed=7)
    a, z = c.bt.cache(lib), c.to.cache(lib)
    call = lambda: lib.tiga_mp_cache_evict(a, c.weights, z, c.to_weights, keep=130, recent=20)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call()
    for lens in ([300, 100, 200], [131, 0, 130], [1, 290, 17], [300, 100, 200]):
        c.bt.length.copy_(torch.tensor(lens, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        replay = [t.clone() for t in (got, c.to.k, c.to.v, c.to_weights, z.length)]
        want = call()
        torch.cuda.synchronize()
        assert torch.equal(replay[0], want) and torch.equal(replay[4], z.length)
        assert same(replay[1], c.to.k) and same(replay[2], c.to.v) and same(replay[3], c.to_weights)


def test_two_calls_at_once(lib):
    """On two streams, each with its own workspace."""
    one, two = (Case([3000, 2000], 2, 64, 16, F16, 1000, 20, "few", seed=s) for s in (8, 9))
    want = [c.expected() for c in (one, two)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for c, s in zip((one, two), streams):
        with torch.cuda.stream(s):
            got.append(lib.tiga_mp_cache_evict(c.bt.cache(lib), c.weights, c.to.cache(lib), c.to_weights, keep=1000, recent=20))
    torch.cuda.synchronize()
    for c, g, (kept, k, v, w) in zip((one, two), got, want):
        assert torch.equal(g.cpu(), kept) and same(c.to.k, k) and same(c.to.v, v) and same(c.to_weights, w)
