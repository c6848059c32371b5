"""Attention behind shared prefixes against 64 bits on the CPU (bounds in relattn_ref) and against the paged call."""
import pytest
import torch

from tests import relattn_ref as R
from tests.paged_ref import Batch
from tests.test_gpu_paged_attention import reference

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


class Grouped(Batch):
    """groups: (sequences, shared positions) of each; sequences past the last group belong to none.  The shared positions
    of a group hold its first sequence's keys and values: whole pages are the same page (or, with `copies`, others)."""

    def __init__(self, lens, groups, kv_heads, width, page, dt, copies=False, before=0, **kw):
        super().__init__(lens, kv_heads, width, page, dt, **kw)
        ptr = [before]
        for n, p in groups:
            first = ptr[-1]
            for b in range(first + 1, first + n):
                for e in range(-(-p // page)):
                    rows = min(page, p - e * page)
                    if rows == page and not copies:
                        self.table[b, e] = self.table[first, e]
                    else:
                        src, dst = int(self.table[first, e]), int(self.table[b, e])
                        self.k[dst, :, :rows], self.v[dst, :, :rows] = self.k[src, :, :rows], self.v[src, :, :rows]
            ptr.append(first + n)
        ints = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
        self.group_ptr, self.group_len = ints(ptr), ints([p for _, p in groups])


def run(lib, bt, q, layout="hnd", **kw):
    return lib.tiga_mp_attention_prefix_fwd(bt.cache(lib), q, bt.dst_ptr, bt.group_ptr, bt.group_len, layout=layout, **kw)


def compare(lib, bt, heads, what, layout="hnd", scale=None):
    q = bt.tokens(heads, layout == "nhd")
    y, lse = run(lib, bt, q, layout, want_lse=True, scale=scale)
    torch.cuda.synchronize()
    if layout == "nhd":
        q, y = q.permute(1, 0, 2), y.permute(1, 0, 2)
    ry, rl, by, bl = reference(bt, q, bt.width ** -0.5 if scale is None else scale)
    n = bt.rows
    R.assert_within(lse[:, :n], rl[:, :n], bl[:, :n], what + " lse")
    R.assert_within(y[:, :n], ry[:, :n], by[:, :n], what + " y")


# lengths (with the new tokens, new tokens), groups (sequences, shared), heads, source heads, width, page, type
CASES = [
    ([(140, 1), (129, 1)], [(2, 128)], 1, 1, 64, 16, F16),
    ([(600, 1), (513, 1), (520, 1), (900, 1)], [(4, 512)], 4, 2, 128, 16, BF16),
    ([(600, 1), (513, 1), (520, 1), (900, 1)], [(4, 500)], 8, 1, 64, 16, F16),           # not whole pages or tiles
    ([(300, 1)] * 40, [(40, 256)], 4, 1, 128, 64, BF16),                                  # wide tiles of shared positions
    ([(1000 + i, 1) for i in range(70)], [(30, 900), (40, 700)], 2, 1, 64, 32, F16),      # two groups, more than 64 sequences
    ([(200 + 3 * i, 1) for i in range(9)], [(3, 128), (1, 200), (2, 199)], 4, 2, 128, 16, BF16),  # one alone, three of no group
    ([(700, 5), (650, 1), (690, 3), (660, 0), (655, 8)], [(5, 640)], 6, 2, 64, 64, F16),  # drafts; one without new tokens
    ([(900, 200), (800, 140), (850, 1)], [(3, 600)], 4, 4, 128, 128, BF16),               # chunks: both passes wide
    ([(400, 1), (300, 1), (50, 1)], [(2, 0), (1, 30)], 4, 2, 64, 16, BF16),               # nothing shared
    ([(5000, 1), (4100, 2), (4097, 1)], [(3, 4096)], 16, 2, 128, 16, F16),
    ([(2100, 1)] * 6, [(6, 2048)], 3, 3, 64, 1024, BF16),                                 # pages longer than a tile
    ([(300, 1), (290, 2)], [(2, 280)], 2, 1, 64, 4, F16),                                 # pages shorter than a load
    ([(1, 1), (1, 1)], [(2, 0)], 1, 1, 128, 16, F16),
]


@pytest.mark.parametrize("lens,groups,H,Hk,D,page,dt", CASES)
@pytest.mark.parametrize("copies", [False, True])
def test_against_64_bits(lib, lens, groups, H, Hk, D, page, dt, copies):
    bt = Grouped(lens, groups, Hk, D, page, dt, copies=copies, seed=len(lens) + page)
    bt.spoil_unused()
    lib.tiga_prefix_validate(bt.cache(lib), bt.num_dst, bt.dst_ptr, bt.group_ptr, bt.group_len)
    compare(lib, bt, H, f"{(len(lens), lens[0], groups, H, Hk, D, page)}")


@pytest.mark.parametrize("before", [1, 2])
def test_sequences_before_the_first_group(lib, before):
    lens = [(50, 1), (300, 4), (400, 1), (390, 1)]
    groups = [(len(lens) - before, 256 if before == 1 else 380)]
    bt = Grouped(lens, groups, 2, 64, 16, BF16, before=before, seed=3)
    compare(lib, bt, 4, "before", layout="nhd", scale=0.2)


def test_no_groups(lib):
    bt = Grouped([(50, 1), (300, 4)], [], 2, 64, 16, BF16, seed=4)
    q = bt.tokens(4)
    y, lse = run(lib, bt, q, want_lse=True)
    z, lse2 = lib.tiga_mp_attention_paged_fwd(bt.cache(lib), q, bt.dst_ptr, want_lse=True)
    torch.cuda.synchronize()
    assert torch.equal(y, z) and torch.equal(lse, lse2)


@pytest.mark.parametrize("lens,shared", [([(300, 1), (290, 1)], 256), ([(300, 40), (290, 17)], 200)])
def test_in_the_queries_place_and_rows_behind(lib, lens, shared):
    bt = Grouped(lens, [(2, shared)], 2, 64, 16, F16, seed=5, tail=7)
    q = bt.tokens(4)
    want = run(lib, bt, q)
    kept = q[:, bt.rows:].clone()
    out = run(lib, bt, q, y=q)
    torch.cuda.synchronize()
    assert out is q and torch.equal(q[:, :bt.rows], want[:, :bt.rows]) and torch.equal(q[:, bt.rows:], kept)


@pytest.mark.parametrize("new", [1, 40])
def test_first_new_token_among_the_shared_positions(lib, new):
    """NaN for that sequence; the others as ever; refused by the validation."""
    bt = Grouped([(300, new), (320, new), (340, new)], [(3, 256)], 1, 64, 16, BF16, seed=6)
    q = bt.tokens(2)
    good = run(lib, bt, q)
    bt.length[1] = 128 + new - 1
    y, lse = run(lib, bt, q, want_lse=True)
    torch.cuda.synchronize()
    p = bt.ptr
    assert torch.isnan(y[:, p[1]:p[2]]).all() and torch.isnan(lse[:, p[1]:p[2]]).all()
    for b in (0, 2):
        R.assert_within(y[:, p[b]:p[b + 1]], good[:, p[b]:p[b + 1]].double().cpu(),
                        2 * reference(bt, q, 0.125)[2][:, p[b]:p[b + 1]], "the others")
    with pytest.raises(lib.TigaError) as e:
        lib.tiga_prefix_validate(bt.cache(lib), bt.num_dst, bt.dst_ptr, bt.group_ptr, bt.group_len)
    assert e.value.code == lib.TIGA_EGRAPH


@pytest.mark.parametrize("new", [1, 40])
def test_bad_pages(lib, new):
    """A shared page that the cache does not have makes its group NaN, one of a sequence's own that sequence."""
    bt = Grouped([(300, new), (320, new), (340, new), (200, new)], [(3, 256)], 1, 128, 16, F16, seed=7)
    q = bt.tokens(2)
    good, table, p = run(lib, bt, q), bt.table.clone(), bt.ptr
    for at, hit in (((0, 3), (0, 1, 2)), ((1, 17), (1,)), ((3, 2), (3,))):
        bt.table.copy_(table)
        bt.table[at] = bt.num_pages
        y, lse = run(lib, bt, q, want_lse=True)
        torch.cuda.synchronize()
        for b in range(4):
            rows = slice(p[b], p[b + 1])
            assert torch.isnan(y[:, rows]).all() if b in hit else torch.equal(y[:, rows], good[:, rows]), (at, b)
            assert bool(torch.isnan(lse[:, rows]).all()) == (b in hit)


@pytest.mark.parametrize("what,code", [("order", -2), ("past", -2), ("negative", -2)])
def test_validation(lib, what, code):
    bt = Grouped([(300, 1), (320, 1), (340, 1)], [(1, 20), (2, 256)], 1, 64, 16, BF16, seed=8)
    check = lambda: lib.tiga_prefix_validate(bt.cache(lib), bt.num_dst, bt.dst_ptr, bt.group_ptr, bt.group_len)
    check()
    if what == "negative":
        bt.group_len[0] = -1
    else:
        bt.group_ptr[1] = 3 if what == "order" else 4
        bt.group_ptr[2] = 2 if what == "order" else 3
    with pytest.raises(lib.TigaError) as e:
        check()
    assert e.value.code == code


def test_groups_out_of_range_stay_inside(lib):
    """Nothing is promised about such a call but that it stays within the tensors and ends."""
    bt = Grouped([(300, 1), (320, 1), (340, 3)], [(1, 20), (2, 256)], 1, 64, 16, BF16, seed=9)
    q = bt.tokens(2)
    for ptr, n in (([0, 3, 1], [1 << 30, -5]), ([-7, 1 << 30, 0], [1 << 30, 1 << 30]), ([3, 3, 3], [9, 9]), ([2, 0, 3], [300, 300])):
        bt.group_ptr.copy_(torch.tensor(ptr, dtype=torch.int32))
        bt.group_len.copy_(torch.tensor(n, dtype=torch.int32))
        run(lib, bt, q)
        torch.cuda.synchronize()


def test_infinite_and_nan_values_of_later_drafts(lib):
    """A value that is not finite reaches the rows that see it, not those before it."""
    bt = Grouped([(300, 5), (320, 4)], [(2, 256)], 1, 64, 16, F16, seed=10)
    q = bt.tokens(2)
    good = run(lib, bt, q)
    page, row = int(bt.table[0, 298 // 16]), 298 % 16      # the fourth of the five
    bt.v[page, 0, row] = float("inf")
    y = run(lib, bt, q)
    torch.cuda.synchronize()
    assert torch.equal(y[:, :3], good[:, :3]) and torch.equal(y[:, 5:], good[:, 5:])
    assert not torch.isfinite(y[:, 3:5]).any()


def test_captured(lib):
    """Lengths, groups and shared positions that change between replays."""
    lens = [(700, 1), (650, 3), (690, 1), (660, 1), (655, 2)]
    bt = Grouped(lens, [(2, 512), (3, 640)], 2, 128, 16, BF16, seed=11)
    q = bt.tokens(8)
    cache = bt.cache(lib)
    call = lambda: lib.tiga_mp_attention_prefix_fwd(cache, q, bt.dst_ptr, bt.group_ptr, bt.group_len, want_lse=True)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, lse = call()
    n = bt.length.clone()
    for ptr, shared, less in (([0, 2, 5], [512, 640], 0), ([0, 0, 5], [9, 512], 3), ([2, 4, 5], [640, 70], 1), ([0, 2, 5], [512, 640], 0)):
        bt.group_ptr.copy_(torch.tensor(ptr, dtype=torch.int32))
        bt.group_len.copy_(torch.tensor(shared, dtype=torch.int32))
        bt.length.copy_(n - less)
        graph.replay()
        torch.cuda.synchronize()
        z, lse2 = call()
        torch.cuda.synchronize()
        assert torch.equal(y, z) and torch.equal(lse, lse2)


@pytest.mark.parametrize("left", [0, 1, 300, 511])
@pytest.mark.parametrize("new", [1, 30])
def test_a_first_sequence_that_has_ended(lib, left, new):
    """What it no longer has is read from the others' own pages."""
    bt = Grouped([(600, 0), (700, new), (650, new), (900, new)], [(4, 512)], 2, 64, 16, F16, copies=True, seed=31)
    bt.length[0] = left
    bt.table[0, -(-left // 16):] = -1
    lib.tiga_prefix_validate(bt.cache(lib), bt.num_dst, bt.dst_ptr, bt.group_ptr, bt.group_len)
    compare(lib, bt, 4, f"ended at {left}")
