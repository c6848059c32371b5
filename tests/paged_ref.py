"""A paged cache for tests: random page order, unequal lengths, and its sequences gathered whole."""
import torch


class Batch:
    """lens: (length with the new tokens, new tokens) of each sequence."""

    def __init__(self, lens, kv_heads, width, page, dt, seed=0, rows_first=False, spare=2, tail=0):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.page, self.kv_heads, self.width, self.dt = lens, page, kv_heads, width, dt
        need = [max(0, -(-n // page)) for n, _ in lens]
        self.num_pages = sum(need) + spare
        order = torch.randperm(self.num_pages, generator=g).to(torch.int32)
        self.table = torch.full((len(lens), max(need + [0]) + 1), -1, dtype=torch.int32)
        at = 0
        for b, c in enumerate(need):
            self.table[b, :c] = order[at:at + c]
            at += c
        shape = (self.num_pages, page, kv_heads, width) if rows_first else (self.num_pages, kv_heads, page, width)
        make = lambda: torch.randn(*shape, generator=g).to(dt)
        view = lambda t: t.permute(0, 2, 1, 3) if rows_first else t
        self.k, self.v = view(make().cuda()), view(make().cuda())
        ptr = [0]
        for _, c in lens:
            ptr.append(ptr[-1] + c)
        self.rows, self.ptr = ptr[-1], ptr
        self.num_dst = self.rows + tail        # rows behind the last sequence
        self.dst_ptr = torch.tensor(ptr, dtype=torch.int32, device="cuda")
        self.length = torch.tensor([n for n, _ in lens], dtype=torch.int32, device="cuda")
        self.table = self.table.cuda()
        self.g = g

    def cache(self, lib):
        return lib.KvCache(self.k, self.v, self.table, self.length)

    def tokens(self, heads, rows_first=False):
        """New rows [heads, rows, width] ("hnd"), or the same packed rows first."""
        t = torch.randn(self.num_dst, heads, self.width, generator=self.g).to(self.dt).cuda()
        return t if rows_first else t.permute(1, 0, 2).contiguous()

    def gathered(self, b):
        """Keys and values [kv_heads, length, width] of sequence b on the CPU, in the cache's type."""
        n = max(0, self.lens[b][0])
        ids = self.table[b, : -(-n // self.page)].long().cpu()
        pick = lambda t: t.cpu()[ids].permute(1, 0, 2, 3).reshape(self.kv_heads, -1, self.width)[:, :n]
        return pick(self.k), pick(self.v)

    def spoil_unused(self):
        """NaN and infinities in every place that no sequence uses."""
        for t, bad in ((self.k, float("nan")), (self.v, float("inf"))):
            keep = torch.zeros(self.num_pages, self.page, dtype=torch.bool)
            for b, (n, _) in enumerate(self.lens):
                for p in range(max(0, n)):
                    keep[int(self.table[b, p // self.page]), p % self.page] = True
            t.masked_fill_(~keep[:, None, :, None].cuda(), bad)
