"""The operators as a server and a trainer use them together: whole prompts packed, their keys and values appended to a cache
whose sequences share an instruction, next tokens behind it, the weights that cached positions get, the eviction of the least,
and tokens after it; and a training step through rotary positions and packed attention."""
import pytest
import torch

from tests import packed_ref as P
from tests import relattn_ref as R

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


class Server:
    """Sequences that begin with the same `shared` tokens; fixed projections of every token."""

    def __init__(self, lib, shared, own, steps, H, Hk, D, dt, page=16, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.lib, self.shared, self.own, self.H, self.Hk, self.D, self.dt, self.page = lib, shared, own, H, Hk, D, dt, page
        B, self.steps = len(own), steps
        self.total = [shared + n + steps for n in own]
        first = [torch.randn(shared, h, D, generator=g).to(dt) for h in (H, Hk, Hk)]
        self.qkv = [[torch.cat([f, torch.randn(n - shared, f.shape[1], D, generator=g).to(dt)]).cuda() for f in first] for n in self.total]
        self.rot = lib.Rotary(lib.tiga_rotary_frequencies(D).cuda())
        whole, need = shared // page, [-(-n // page) for n in self.total]
        pages = whole + sum(n - whole for n in need)
        order = torch.randperm(pages, generator=g).to(torch.int32)
        self.table = torch.full((B, max(need)), -1, dtype=torch.int32)
        at = whole
        for b, n in enumerate(need):
            self.table[b, :whole] = order[:whole]            # the instruction's whole pages are stored once
            self.table[b, whole:n] = order[at:at + n - whole]
            at += n - whole
        ints = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
        self.ints = ints
        self.k, self.v = (torch.randn(pages, Hk, page, D, generator=g).to(dt).cuda() for _ in "kv")
        self.length = ints([shared + n for n in own])
        self.cache = lib.KvCache(self.k, self.v, self.table.cuda(), self.length)
        self.group = ints([0, B]), ints([shared])

    def prompts(self):
        """Every prompt whole, packed: attention, and its keys and values into the pages."""
        lib, lens = self.lib, [self.shared + n for n in self.own]
        ptr = [0]
        for n in lens:
            ptr.append(ptr[-1] + n)
        pos = torch.cat([torch.arange(n) for n in lens]).to(torch.int32).cuda()
        q, k, v = (torch.cat([t[i][:n] for t, n in zip(self.qkv, lens)]) for i in range(3))
        q, k = (lib.tiga_mp_rotary_fwd(t, pos, self.rot, layout="nhd") for t in (q, k))
        ptr = self.ints(ptr)
        y = lib.tiga_mp_attention_packed_fwd(q, k, v, ptr, layout="nhd")
        # rotated already; the shared pages are the first sequence's to write
        whole, rows, new = self.shared // self.page * self.page, [], [0]
        for b, n in enumerate(lens):
            rows.append(torch.arange(whole if b else 0, n) + int(ptr[b]))
            new.append(new[-1] + rows[-1].numel())
        rows = torch.cat(rows).cuda()
        lib.tiga_mp_cache_append(self.cache, k[rows], v[rows], self.ints(new), layout="nhd")
        return q, k, v, y, ptr

    def token(self, step):
        """The next token of every sequence, as a server feeds it."""
        lib = self.lib
        self.length += 1
        q, k, v = (torch.stack([t[i][self.shared + n + step] for t, n in zip(self.qkv, self.own)]) for i in range(3))
        ptr = torch.arange(len(self.own) + 1, dtype=torch.int32, device="cuda")
        q = lib.tiga_mp_cache_append(self.cache, k, v, ptr, self.rot, q=q, layout="nhd")
        y, lse = lib.tiga_mp_attention_prefix_fwd(self.cache, q, ptr, *self.group, want_lse=True, layout="nhd")
        return q, y, lse, ptr


def turned(s, b, i, n):
    """Rows 0 .. n of sequence b's queries (0) or keys (1), rotated, as the cache holds them."""
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    return s.lib.tiga_mp_rotary_fwd(s.qkv[b][i][:n].contiguous(), pos, s.rot, layout="nhd")


@pytest.mark.parametrize("shared,own,H,Hk,D,dt", [(150, [40, 7, 120], 4, 2, 64, F16), (300, [100, 33], 8, 1, 128, BF16)])
def test_prompts_tokens_and_eviction(lib, shared, own, H, Hk, D, dt):
    steps, B = 6, len(own)
    s = Server(lib, shared, own, steps, H, Hk, D, dt)
    scale = D ** -0.5
    q, k, v, y, ptr = s.prompts()
    torch.cuda.synchronize()
    for b in range(B):
        here = slice(int(ptr[b]), int(ptr[b + 1]))
        n = here.stop - here.start
        for h in range(H):
            j = h * Hk // H
            f = R.rows(*(t[here, i].double().cpu() for t, i in ((q, h), (k, j), (v, j))), torch.ones(n, n).tril().bool(), scale)
            R.assert_within(y[here, h], f["y"], f["y_bound"](dt), "prompt")

    # next tokens; the weights of a cache without shared pages, which a copy has
    expected = [[torch.zeros(2, 0, dtype=torch.float64) for _ in range(Hk)] for _ in range(B)]   # and what they may be off by
    lib.tiga_prefix_validate(s.cache, B, torch.arange(B + 1, dtype=torch.int32, device="cuda"), *s.group)
    need = [-(-n // s.page) for n in s.total]
    table = torch.full((B, max(need)), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = torch.arange(at, at + n)
        at += n
    alone = lib.KvCache(torch.zeros(at, *s.k.shape[1:], dtype=dt, device="cuda"), torch.zeros(at, *s.k.shape[1:], dtype=dt, device="cuda"),
                        table.cuda(), s.length)
    for b, n in enumerate(need):
        alone.k_pages[table[b, :n].long()] = s.k[s.table[b, :n].long()]
        alone.v_pages[table[b, :n].long()] = s.v[s.table[b, :n].long()]
    weights = torch.zeros(at, Hk, s.page, device="cuda")
    for step in range(steps - 1):
        q, y, lse, one = s.token(step)
        for b in range(B):                                    # the token's own row, as append stored it
            p = shared + own[b] + step
            for a, t in ((alone.k_pages, s.k), (alone.v_pages, s.v)):
                a[table[b, p // s.page], :, p % s.page] = t[s.table[b, p // s.page], :, p % s.page]
        lib.tiga_mp_cache_weights(alone, q, lse, one, weights, decay=0.5, layout="nhd")
        torch.cuda.synchronize()
        for b in range(B):
            n = shared + own[b] + step + 1
            kk, vv = turned(s, b, 1, n), s.qkv[b][2][:n]
            given = [torch.zeros(2, n, dtype=torch.float64) for _ in range(Hk)]
            for h in range(H):
                j = h * Hk // H
                f = R.rows(q[b:b + 1, h].double().cpu(), kk[:, j].double().cpu(), vv[:, j].double().cpu(), torch.ones(1, n).bool(), scale)
                R.assert_within(y[b:b + 1, h], f["y"], f["y_bound"](dt), "next token")
                R.assert_within(lse[h, b:b + 1], f["lse"], f["lse_bound"], "next token's lse")
                # a weight is off by its score's error, by lse's, and by the roundings of lse * log2 e and the argument
                off = 2 * f["es"][0] + 2 * f["lse_bound"] + 2.0 ** -22 * (f["lse"].abs() + 1)
                given[j] += torch.stack([f["p"][0], f["p"][0] * off])
            for j in range(Hk):
                old = expected[b][j] if step else torch.zeros(2, n - 1, dtype=torch.float64)
                new = torch.cat([old * 0.5, torch.zeros(2, 1, dtype=torch.float64)], 1) + given[j]
                new[1] += (R.sums(H // Hk) + 2.0 ** -22) * new[0]     # the sum's own rounding
                expected[b][j] = new
    for b in range(B):
        n = shared + own[b] + steps - 1
        place = torch.arange(n)
        got = weights[table[b].long()[place // s.page], :, place % s.page].double().cpu()
        for j in range(Hk):
            R.assert_within(got[:, j], *expected[b][j], "weights")

    # keep two thirds, the last tokens among them, and go on
    keep = 2 * (shared + min(own)) // 3
    small = [-(-keep // s.page) + 1] * B
    to_table = torch.arange(sum(small), dtype=torch.int32).view(B, -1)
    to = lib.KvCache(torch.zeros(sum(small), *s.k.shape[1:], dtype=dt, device="cuda"), torch.zeros(sum(small), *s.k.shape[1:], dtype=dt, device="cuda"),
                     to_table.cuda(), torch.zeros(B, dtype=torch.int32, device="cuda"))
    to_weights = torch.zeros(sum(small), Hk, s.page, device="cuda")
    kept = lib.tiga_mp_cache_evict(alone, weights, to, to_weights, keep=keep, recent=8)
    true_pos = s.length.clone()
    to.length += 1
    q, k, v = (torch.stack([t[i][shared + n + steps - 1] for t, n in zip(s.qkv, own)]) for i in range(3))
    q, k = (lib.tiga_mp_rotary_fwd(t.view(1, B, -1, D), true_pos.view(1, B), s.rot, layout="bnhd").view(B, -1, D) for t in (q, k))
    one = torch.arange(B + 1, dtype=torch.int32, device="cuda")
    lib.tiga_mp_cache_append(to, k, v, one, layout="nhd")
    y, lse = lib.tiga_mp_attention_paged_fwd(to, q, one, want_lse=True, layout="nhd")
    lib.tiga_mp_cache_weights(to, q, lse, one, to_weights, layout="nhd")
    torch.cuda.synchronize()
    assert to.length.tolist() == [keep + 1] * B
    for b in range(B):
        n = shared + own[b] + steps
        kk, vv = turned(s, b, 1, n), s.qkv[b][2][:n]
        for h in range(H):
            j = h * Hk // H
            stay = torch.cat([kept[b, j].long(), torch.tensor([n - 1], device="cuda")])
            assert (stay[1:] > stay[:-1]).all() and (stay[-9:] == torch.arange(n - 9, n, device="cuda")).all()
            f = R.rows(q[b:b + 1, h].double().cpu(), kk[stay, j].double().cpu(), vv[stay, j].double().cpu(), torch.ones(1, keep + 1).bool(), scale)
            R.assert_within(y[b:b + 1, h], f["y"], f["y_bound"](dt), "after eviction")
            R.assert_within(lse[h, b:b + 1], f["lse"], f["lse_bound"], "lse after eviction")
        total = float(to_weights[to_table[b].long()].sum())
        assert total > 0 and torch.isfinite(to_weights).all()


def test_training_step_through_rotary_and_packed_attention(lib):
    """Gradients through both operators chained by autograd against 64 bits."""
    s = P.Packed([33, 1, 90], 4, 2, 64, F16, seed=4)
    pos = torch.cat([torch.arange(n) for n in s.lens]).to(torch.int32).cuda()
    rot = lib.Rotary(lib.tiga_rotary_frequencies(64).cuda())
    x, k = (t.clone().requires_grad_(True) for t in (s.q, s.k))
    v = s.v.clone().requires_grad_(True)
    q2, k2 = lib.rotary(x, pos, rot, layout="hnd"), lib.rotary(k, pos, rot, layout="hnd")
    q2.retain_grad()
    k2.retain_grad()
    y = lib.packed_attention(q2, k2, v, s.ptr_t)
    y.backward(s.dy)
    s.q, s.k = q2.detach(), k2.detach()
    out, bound = P.reference(s, 64 ** -0.5)
    for t, name in ((q2, "dq"), (k2, "dk"), (v, "dv")):
        R.assert_within(t.grad, out[name], bound[name], name)
    for leaf, inner in ((x, q2), (k, k2)):
        assert torch.equal(leaf.grad, lib.tiga_mp_rotary_bwd(inner.grad, pos, rot, layout="hnd"))


def test_a_server_step_captured(lib):
    """Append, attention behind the shared prefix, weights and an eviction in one graph; lengths advance between replays."""
    B, H, Hk, D, page, dt = 3, 4, 2, 64, 16, BF16
    g = torch.Generator().manual_seed(6)
    t = lambda *a: torch.randn(*a, generator=g).to(dt).cuda()
    per = 30
    pages = [t(B * per, Hk, page, D) for _ in range(4)]
    table = torch.randperm(B * per, generator=g).to(torch.int32).view(B, per).cuda()
    length = torch.tensor([300, 350, 280], dtype=torch.int32, device="cuda")
    for b in (1, 2):                                          # 256 shared positions, in copies
        for p in pages:
            p[table[b, :16].long()] = p[table[0, :16].long()]
    to_k, to_v = t(B * 8, Hk, page, D), t(B * 8, Hk, page, D)
    to_table = torch.arange(B * 8, dtype=torch.int32, device="cuda").view(B, 8)
    group = torch.tensor([0, B], dtype=torch.int32, device="cuda"), torch.tensor([256], dtype=torch.int32, device="cuda")
    ptr = torch.arange(B + 1, dtype=torch.int32, device="cuda")
    q, k, v = t(B, H, D), t(B, Hk, D), t(B, Hk, D)
    rot = lib.Rotary(lib.tiga_rotary_frequencies(D).cuda())

    def make(k_pages, v_pages):
        cache = lib.KvCache(k_pages, v_pages, table, length)
        to = lib.KvCache(to_k.clone(), to_v.clone(), to_table, torch.zeros_like(length))
        weights, to_weights = torch.ones(B * per, Hk, page, device="cuda"), torch.zeros(B * 8, Hk, page, device="cuda")

        def step():
            qr = lib.tiga_mp_cache_append(cache, k, v, ptr, rot, q=q, layout="nhd")
            y, lse = lib.tiga_mp_attention_prefix_fwd(cache, qr, ptr, *group, want_lse=True, layout="nhd")
            lib.tiga_mp_cache_weights(cache, qr, lse, ptr, weights, decay=0.9, layout="nhd")
            kept = lib.tiga_mp_cache_evict(cache, weights, to, to_weights, keep=120, recent=10)
            return y, lse, kept, weights, to.k_pages, to.v_pages, to_weights, to.length

        return step

    first, second = make(pages[0], pages[1]), make(pages[0].clone(), pages[1].clone())
    state = [x.clone() for x in (pages[0], pages[1])]
    first()                                                   # allocations and the library's first calls
    torch.cuda.synchronize()
    pages[0].copy_(state[0])
    pages[1].copy_(state[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = first()
    out[3].fill_(1.0)                                         # the weights, as the second starts
    for i in range(4):
        for a in (q, k, v):
            a.copy_(torch.randn(a.shape, generator=g).to(dt))
        graph.replay()
        want = second()
        torch.cuda.synchronize()
        for n, (a, b) in enumerate(zip(out, want)):
            assert torch.equal(a, b), (i, n)
        length += 1
