"""Prompts packed into one batch, and a cache that is shared and kept small, as measurable cases.

Four operators: causal attention of packed sequences of different lengths with heads that share sources (a forward,
and a training step with the gradients of q, k and v), attention of new tokens over a paged cache of which groups of
sequences share their first positions, the accumulation of the weights that cached positions get, and the eviction of
the positions with the least weight.

With ``own`` false a pass is elementary torch operations in 32 bits, rounded once; with ``own`` true it is the calls of
``paper_2609_24802_amd.binding``.  ``exact`` is the definition in 64 bits.
"""
import math
import random

import torch

own = False

DEV = "cuda:0"


def listed():
    return [
        # three short questions, whole: latency
        dict(name="packed_tiny", op="packed", batch=3, rows=37, heads=16, kv_heads=4, width=64, dtype="f16", step=False),
        # prompts of a serving batch, lengths between a few and thousands
        dict(name="packed_prompts", op="packed", batch=17, rows=16384, heads=32, kv_heads=8, width=128, dtype="bf16",
             step=False),
        # training on short documents packed without padding
        dict(name="packed_short_step", op="packed", batch=61, rows=8001, heads=16, kv_heads=16, width=64, dtype="f16",
             step=True),
        # training on long documents, four heads to a source head; the largest
        dict(name="packed_long_step", op="packed", batch=3, rows=16384, heads=16, kv_heads=4, width=128, dtype="bf16",
             step=True),
        # next tokens of a few users behind one short instruction: latency
        dict(name="prefix_token_4", op="prefix", batch=4, groups=1, heads=16, kv_heads=4, width=64, page=16, shared=500,
             longest=200, chunk=1, dtype="bf16"),
        # next tokens of a serving batch whose prompts begin with the same instructions and examples
        dict(name="prefix_token_64", op="prefix", batch=64, groups=1, heads=32, kv_heads=8, width=128, page=16,
             shared=8192, longest=1000, chunk=1, dtype="bf16"),
        # questions about four long documents, a few drafted tokens each to be checked
        dict(name="prefix_drafts", op="prefix", batch=24, groups=4, heads=16, kv_heads=2, width=128, page=64,
             shared=40000, longest=700, chunk=5, dtype="f16"),
        # next tokens of a serving batch: what every cached position has been worth so far
        dict(name="weights_token_64", op="weights", batch=64, heads=32, kv_heads=8, width=128, page=16, longest=8192,
             chunk=1, chunks=0, dtype="bf16"),
        # the last tokens of a long prompt look back over it
        dict(name="weights_chunk", op="weights", batch=5, heads=16, kv_heads=4, width=128, page=64, longest=9000,
             chunk=1023, chunks=2, dtype="f16"),
        # one short conversation over its budget
        dict(name="evict_one", op="evict", batch=1, kv_heads=4, width=64, page=16, longest=545, keep=512, recent=64,
             dtype="f16"),
        # a serving batch over its budget
        dict(name="evict_batch", op="evict", batch=64, kv_heads=8, width=128, page=16, longest=2500, keep=2048,
             recent=256, dtype="bf16"),
        # long prompts reduced to what their last tokens looked at
        dict(name="evict_long", op="evict", batch=2, kv_heads=8, width=128, page=64, longest=131072, keep=16384,
             recent=1000, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["packed", "packed", "packed", "prefix", "prefix", "weights", "evict"])
    case = dict(op=op, width=rng.choice([64, 128]), dtype=rng.choice(["f16", "bf16"]))
    case["kv_heads"] = _log(rng, 1, 16)
    if op != "evict":
        case["heads"] = case["kv_heads"] * rng.choice([1, 1, 2, 4, 8])
    if op == "packed":
        case["step"] = rng.random() < 0.6
        case["rows"] = _log(rng, 1, 16384)
        case["batch"] = _log(rng, 1, min(64, case["rows"]))
        # at most the pairs of the largest, whatever the lengths
        while case["rows"] ** 2 * case["heads"] * case["width"] > 10000 ** 2 * 16 * 128:
            case["rows"] = case["rows"] * 3 // 4
        case["batch"] = min(case["batch"], case["rows"])
        return case
    case["page"], case["batch"] = rng.choice([16, 32, 64, 128]), _log(rng, 1, 64)
    if op == "prefix":
        case["groups"] = rng.randint(1, min(4, case["batch"]))
        case["shared"], case["longest"] = _log(rng, 16, 40000), _log(rng, 8, 2000)
        case["chunk"] = rng.choice([1, 1, _log(rng, 2, 8)])
        while (case["batch"] * (case["shared"] + case["longest"]) * case["kv_heads"] * case["width"] > 64 * 9192 * 8 * 128
               or case["batch"] * (case["shared"] + case["longest"]) * case["heads"] * case["chunk"] > 24 * 40700 * 16 * 5):
            big = "shared" if case["shared"] > 8 * case["longest"] else "batch" if case["batch"] > 4 else "longest"
            case[big] = max(1, case[big] * 2 // 3)
        case["groups"] = min(case["groups"], case["batch"])
        case["longest"] = max(case["longest"], case["chunk"])
        return case
    if op == "weights":
        case["longest"] = _log(rng, 20, 32768)
        case["chunk"], case["chunks"] = 1, 0
        if rng.random() < 0.5:
            case["chunk"], case["chunks"] = _log(rng, 2, min(2048, case["longest"])), rng.randint(1, min(3, case["batch"]))
        while (case["batch"] * case["longest"] * case["kv_heads"] * case["width"] > 64 * 8192 * 8 * 128
               or case["batch"] * case["longest"] * case["heads"] * (case["chunk"] if case["chunks"] else 1) > 5 * 9000 * 16 * 1023):
            big = "batch" if case["batch"] > 4 else "chunk" if case["chunk"] > 64 else "longest"
            case[big] = max(1, case[big] * 2 // 3)
        case["chunk"] = min(case["chunk"], case["longest"])
        case["chunks"] = min(case["chunks"], case["batch"])
        return case
    case["longest"] = _log(rng, 20, 131072)
    while case["batch"] * case["longest"] * case["kv_heads"] * case["width"] > 2 * 131072 * 8 * 128:
        big = "batch" if case["batch"] > 8 else "longest"
        case[big] = max(1, case[big] * 2 // 3)
    case["keep"] = _log(rng, max(1, case["longest"] // 8), case["longest"])
    case["recent"] = rng.choice([0, _log(rng, 1, case["keep"]), case["keep"] // 8])
    return case


# ------------------------------------------------------------------------------------- inputs

_TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


def _packed_lengths(case):
    """Lengths that sum to the rows: spread over the logarithm, one token among them where there are more than two."""
    rng, b, n = random.Random(case["batch"] * 1_000_003 + case["rows"]), case["batch"], case["rows"]
    share = [math.exp(rng.uniform(0.0, 4.0)) for _ in range(b)]
    cut, at = [0], 0.0
    for x in share:
        at += x
        cut.append(int(round(at / sum(share) * (n - b))))
    lens = [cut[i + 1] - cut[i] + 1 for i in range(b)]
    if b > 2:
        lens[0], lens[1] = lens[0] + lens[1] - 1, 1
    return lens


def _cache_lengths(case):
    """(length with the new tokens, new tokens) of each sequence: the longest first, the others spread over the
    logarithm; the first `chunks` of them bring a chunk, the others one token."""
    rng = random.Random(case["batch"] * 1_000_003 + case["longest"])
    out = []
    for b in range(case["batch"]):
        c = case["chunk"] if b < case["chunks"] else 1
        n = case["longest"] if b == 0 else _log(rng, max(1, case["longest"] / 16), case["longest"])
        out.append((max(n, c), c))
    return out


def _evict_lengths(case):
    """The longest first, the others between just under the budget and the longest: one in eight has nothing to give."""
    rng = random.Random(case["batch"] * 1_000_003 + case["longest"])
    lo = min(case["keep"], case["longest"])
    return [case["longest"]] + [rng.randint(max(1, lo // 2), lo) if b % 8 == 7 else rng.randint(lo, case["longest"])
                                for b in range(1, case["batch"])]


def _shares(case):
    """(shared positions, length with the new tokens, new tokens, group) of each sequence."""
    rng, b, n = random.Random(case["batch"] * 1_000_003 + case["shared"]), case["batch"], case["groups"]
    shared = [case["shared"]] + [_log(rng, max(1, case["shared"] / 4), case["shared"]) for _ in range(n - 1)]
    out = []
    for i in range(b):
        g = i * n // b
        c = case["chunk"] if i % 3 == 0 else rng.randint(1, case["chunk"])
        out.append((shared[g], shared[g] + max(c, _log(rng, max(1, case["longest"] / 16), case["longest"])), c, g))
    return out


def _starts(counts):
    ptr = [0]
    for c in counts:
        ptr.append(ptr[-1] + c)
    return ptr


def _randn(g, dt):
    return lambda *s: torch.randn(*s, generator=g, device=DEV).to(dt)


def _ints(a):
    return torch.tensor(a, dtype=torch.int32, device=DEV)


def _tables(g, need, spare=3, shared=None):
    """The pages of sequences that need so many each, in no order: (table, pages in all).  shared: (first entries that a
    sequence takes from another, that one) of each."""
    shared = shared or [(0, 0)] * len(need)
    pages = sum(n - s for n, (s, _) in zip(need, shared)) + spare
    order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    table = torch.full((len(need), max(need)), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, (n, (s, of)) in enumerate(zip(need, shared)):
        table[b, :s] = table[of, :s]
        table[b, s:n] = order[at:at + n - s]
        at += n - s
    return table, pages


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed) * 7919 + 31)
    randn = _randn(g, _TYPES[case["dtype"]])
    op, w, hk, h = case["op"], case["width"], case["kv_heads"], case.get("heads", 0)
    s = dict(case=case)
    if op == "packed":
        lens = _packed_lengths(case)
        n = case["rows"]
        # the projection's own layout: queries, keys and values of a token side by side
        qkv = randn(n, h + 2 * hk, w)
        s["q"], s["k"], s["v"] = qkv[:, :h], qkv[:, h:h + hk], qkv[:, h + hk:]
        s["lens"], s["ptr"] = lens, _ints(_starts(lens))
        if case["step"]:
            s["dy"] = randn(n, h, w)
            if own:
                for f in ("q", "k", "v"):
                    s[f] = s[f].detach().requires_grad_(True)
        return s
    page = case["page"]
    up = lambda n: -(-n // page)
    if op == "evict":
        lens = _evict_lengths(case)
        table, pages = _tables(g, [up(n) for n in lens])
        to_lens = [min(n, case["keep"]) for n in lens]
        s["to_table"], to_pages = _tables(g, [up(n) for n in to_lens])
        s["to_k"], s["to_v"] = (torch.zeros(to_pages, page, hk, w, dtype=_TYPES[case["dtype"]], device=DEV) for _ in "kv")
        s["to_weights"] = torch.zeros(to_pages, hk, page, device=DEV)
        s["to_length"] = _ints([0] * len(lens))
        # what sums of attention weights look like: a few large ones, many small ones, some of them equal
        x = torch.exp(2.0 * torch.randn(pages, hk, page, generator=g, device=DEV))
        s["weights"] = torch.where(x < 0.5, (x * 64).round() / 64, x)
    else:
        if op == "prefix":
            shares = _shares(case)
            lens, counts = [n for _, n, _, _ in shares], [c for _, _, c, _ in shares]
            first = {}
            for b, (_, _, _, i) in enumerate(shares):
                first.setdefault(i, b)
            table, pages = _tables(g, [up(n) for n in lens], 3, [(0, 0) if first[i] == b else (p // page, first[i])
                                                                 for b, (p, _, _, i) in enumerate(shares)])
            s["group_ptr"] = _ints([first[i] for i in range(len(first))] + [len(lens)])
            s["group_len"] = _ints([shares[first[i]][0] for i in range(len(first))])
        else:
            lens, counts = zip(*_cache_lengths(case))
            table, pages = _tables(g, [up(n) for n in lens])
        ptr = _starts(counts)
        s["ptr"], s["counts"], s["q"] = _ints(ptr), counts, randn(ptr[-1], h, w)
    s["k_pages"], s["v_pages"] = randn(pages, page, hk, w), randn(pages, page, hk, w)
    s["table"], s["length"], s["lens"] = table, _ints(lens), lens
    if op == "prefix":  # a page that is shared in part: its sequences have it each
        for b, (p, _, _, i) in enumerate(shares):
            if p % page and first[i] != b:
                src, dst = table[first[i], p // page], table[b, p // page]
                for t in (s["k_pages"], s["v_pages"]):
                    t[dst, :p % page] = t[src, :p % page]
    if op == "weights":
        s["weights"] = torch.rand(pages, hk, page, generator=g, device=DEV) * 4
        s["out"] = torch.zeros_like(s["weights"])
        seq, place = _plain_rows(s)
        lse = torch.logsumexp(_plain_scores(s)[0], -1)
        s["lse"] = lse.permute(0, 3, 1, 2)[seq, place].reshape(-1, h).t().contiguous()
    if own:
        from paper_2609_24802_amd import binding as tb
        s["cache"] = tb.KvCache(s["k_pages"].permute(0, 2, 1, 3), s["v_pages"].permute(0, 2, 1, 3), table, s["length"])
        if op == "evict":
            s["to"] = tb.KvCache(s["to_k"].permute(0, 2, 1, 3), s["to_v"].permute(0, 2, 1, 3), s["to_table"], s["to_length"])
    return s


# ------------------------------------------------------------------------------ plain passes, 32 bits


def _plain_packed(s):
    case = s["case"]
    n, h, hk, w, dt = case["rows"], case["heads"], case["kv_heads"], case["width"], s["q"].dtype
    scale, g = w ** -0.5, h // hk
    outs = [torch.empty(n, i, w, dtype=dt, device=DEV) for i in ((h, h, hk, hk) if case["step"] else (h,))]
    lse = torch.empty(h, n, device=DEV)
    at = 0
    for c in s["lens"]:  # a sequence at a time: together their scores would not fit
        here = slice(at, at + c)
        at += c
        # [source head, head of its group, token, width]
        rows = lambda t: t[here].float().view(c, hk, g, w).permute(1, 2, 0, 3).reshape(hk, g * c, w)
        back = lambda t: t.view(hk, g, c, w).permute(2, 0, 1, 3).reshape(c, h, w).to(dt)
        q, k, v = rows(s["q"]), s["k"][here].float().transpose(0, 1).contiguous(), s["v"][here].float().transpose(0, 1).contiguous()
        p = torch.matmul(q, k.transpose(1, 2).contiguous()).mul_(scale).view(hk, g, c, c)
        p.masked_fill_(torch.ones(c, c, dtype=torch.bool, device=DEV).triu_(1), -math.inf)
        top = p.amax(-1, keepdim=True)
        p.sub_(top).exp_()
        mass = p.sum(-1, keepdim=True)
        p.div_(mass)
        p = p.view(hk, g * c, c)
        y = torch.matmul(p, v)
        outs[0][here], lse[:, here] = back(y), (mass.log() + top).view(h, c)
        if case["step"]:
            dy = rows(s["dy"])
            dv = torch.matmul(p.transpose(1, 2).contiguous(), dy)
            p.mul_(torch.matmul(dy, v.transpose(1, 2).contiguous()).sub_((dy * y).sum(-1, keepdim=True)))
            outs[1][here] = back(torch.matmul(p, k) * scale)
            outs[2][here] = (torch.matmul(p.transpose(1, 2).contiguous(), q) * scale).transpose(0, 1).to(dt)
            outs[3][here] = dv.transpose(0, 1).to(dt)
    return tuple(outs) if case["step"] else (outs[0], lse)


def _plain_rows(s):
    """Sequence and place within its new tokens of every packed row."""
    counts = (s["ptr"][1:] - s["ptr"][:-1]).long()
    seq = torch.repeat_interleave(torch.arange(counts.numel(), device=DEV), counts, output_size=s["q"].shape[0])
    return seq, torch.arange(s["q"].shape[0], device=DEV) - s["ptr"][seq]


def _plain_cells(table, page, n):
    """Page and row of the positions [0, n) of every sequence."""
    at = torch.arange(n, device=DEV)
    return table[:, at // page].long().clamp_(min=0), at % page


def _plain_scores(s):
    """Scores [batch, source head, head of its group, new token, position] padded to the longest, in fp32; -inf where
    the token does not see the position, or neither is there."""
    case = s["case"]
    hk, w = case["kv_heads"], case["width"]
    g, c, n = case["heads"] // hk, max(s["counts"]), max(s["lens"])
    seq, place = _plain_rows(s)
    q = torch.zeros(len(s["lens"]), c, hk, g, w, device=DEV)
    q[seq, place] = s["q"].float().view(-1, hk, g, w)
    ids, slot = _plain_cells(s["table"], case["page"], n)
    kt = s["k_pages"][ids, slot].permute(0, 2, 3, 1).float().contiguous()
    sc = torch.matmul(q.permute(0, 2, 3, 1, 4).reshape(len(s["lens"]), hk, g * c, w), kt).mul_(w ** -0.5)
    count = s["ptr"][1:] - s["ptr"][:-1]
    last = (s["length"] - count)[:, None] + torch.arange(c, device=DEV)
    last = torch.where(torch.arange(c, device=DEV) < count[:, None], last, -1)
    sc = sc.view(len(s["lens"]), hk, g, c, n)
    sc.masked_fill_((torch.arange(n, device=DEV) > last[:, :, None])[:, None, None], -math.inf)
    return sc, ids, slot


def _plain_prefix(s):
    case = s["case"]
    hk, w, h = case["kv_heads"], case["width"], case["heads"]
    sc, ids, slot = _plain_scores(s)
    b, _, g, c, n = sc.shape
    top = sc.amax(-1, keepdim=True).clamp_(min=-3e38)
    p = sc.sub_(top).exp_()
    mass = p.sum(-1, keepdim=True)
    v = s["v_pages"][ids, slot].transpose(1, 2).float().contiguous()
    y = torch.matmul(p.view(b, hk, g * c, n), v).view(b, hk, g, c, w) / mass
    lse = (mass.log() + top)[..., 0]
    seq, place = _plain_rows(s)
    return (y.permute(0, 3, 1, 2, 4)[seq, place].reshape(-1, h, w).to(s["q"].dtype),
            lse.permute(0, 3, 1, 2)[seq, place].reshape(-1, h).t().contiguous())


def _plain_weights(s):
    hk, h = s["case"]["kv_heads"], s["case"]["heads"]
    sc, ids, slot = _plain_scores(s)
    b, _, g, c, n = sc.shape
    seq, place = _plain_rows(s)
    lse = torch.zeros(b, c, h, device=DEV)
    lse[seq, place] = s["lse"].t()
    got = sc.sub_(lse.view(b, c, hk, g).permute(0, 2, 3, 1)[..., None]).exp_().sum((2, 3))
    at = torch.arange(n, device=DEV)
    old = s["weights"].permute(0, 2, 1)[ids, slot].permute(0, 2, 1)
    fresh = at >= (s["length"] - (s["ptr"][1:] - s["ptr"][:-1]))[:, None]  # new positions had no weight before
    got += torch.where(fresh[:, None], torch.zeros_like(old), old * _DECAY)
    here = at < s["length"][:, None]
    s["out"].permute(0, 2, 1)[ids[here], slot.expand(b, -1)[here]] = got.permute(0, 2, 1)[here]
    return s["out"]


_DECAY = 0.96875  # what earlier weights keep at every call


def _plain_evict(s):
    case = s["case"]
    hk, keep, recent = case["kv_heads"], case["keep"], case["recent"]
    b, n = len(s["lens"]), max(s["lens"])
    ids, slot = _plain_cells(s["table"], case["page"], n)
    at = torch.arange(n, device=DEV)
    rank = s["weights"].permute(0, 2, 1)[ids, slot].permute(0, 2, 1).clone()
    length = s["length"].long()
    rank.masked_fill_((at >= (length - recent)[:, None])[:, None], math.inf)   # the last ones stay
    rank.masked_fill_((at >= length[:, None])[:, None], -math.inf)
    order = rank.sort(dim=-1, descending=True, stable=True).indices[..., : min(keep, n)]
    kept = torch.full((b, hk, keep), -1, dtype=torch.int64, device=DEV)
    left = length.clamp(max=keep)[:, None, None]
    # positions that are not there sort last
    order = torch.where(torch.arange(order.shape[-1], device=DEV) < left, order, n).sort(-1).values
    kept[..., : order.shape[-1]] = torch.where(order < n, order, -1)
    row, head, to = (kept >= 0).nonzero(as_tuple=True)
    src, page = kept[row, head, to], case["page"]
    ids, slot = s["table"][row, src // page].long(), src % page
    to_ids, to_slot = s["to_table"][row, to // page].long(), to % page
    s["to_k"][to_ids, to_slot, head] = s["k_pages"][ids, slot, head]
    s["to_v"][to_ids, to_slot, head] = s["v_pages"][ids, slot, head]
    s["to_weights"][to_ids, head, to_slot] = s["weights"][ids, head, slot]
    s["to_length"].copy_(s["length"].clamp(max=keep))
    return s["to_k"], s["to_v"], s["to_weights"], s["to_length"], kept.to(torch.int32)


# -------------------------------------------------------------------------------------- passes


def _own(s):
    from paper_2609_24802_amd import binding as tb
    case = s["case"]
    op = case["op"]
    if op == "packed":
        if not case["step"]:
            return tb.tiga_mp_attention_packed_fwd(s["q"], s["k"], s["v"], s["ptr"], want_lse=True, layout="nhd")
        y = tb.packed_attention(s["q"], s["k"], s["v"], s["ptr"], layout="nhd")
        return (y,) + torch.autograd.grad(y, (s["q"], s["k"], s["v"]), s["dy"])
    if op == "prefix":
        return tb.tiga_mp_attention_prefix_fwd(s["cache"], s["q"], s["ptr"], s["group_ptr"], s["group_len"], want_lse=True,
                                               layout="nhd")
    if op == "weights":
        return tb.tiga_mp_cache_weights(s["cache"], s["q"], s["lse"], s["ptr"], s["weights"], out=s["out"], decay=_DECAY,
                                        layout="nhd")
    kept = tb.tiga_mp_cache_evict(s["cache"], s["weights"], s["to"], s["to_weights"], keep=case["keep"],
                                  recent=case["recent"])
    return s["to_k"], s["to_v"], s["to_weights"], s["to_length"], kept


def run(s):
    if own:
        return _own(s)
    plain = dict(packed=_plain_packed, prefix=_plain_prefix, weights=_plain_weights, evict=_plain_evict)
    return plain[s["case"]["op"]](s)


def work(case):
    op, w, hk = case["op"], case["width"], case["kv_heads"]
    if op == "packed":
        h, n = case["heads"], float(case["rows"])
        q, kv, pairs = 2.0 * n * h * w, 4.0 * n * hk * w, h * sum(c * (c + 1) / 2.0 for c in _packed_lengths(case))
        if not case["step"]:
            return {"bytes": 2 * q + kv + 4.0 * n * h, "flops": 4.0 * w * pairs}
        return {"bytes": 4 * q + 2 * kv, "flops": 14.0 * w * pairs}  # q, k, v, dy in; y, dq, dk, dv out
    if op == "prefix":
        shares, h = _shares(case), case["heads"]
        q = 2.0 * sum(c for _, _, c, _ in shares) * h * w
        # the shared positions once a group
        kv = 4.0 * hk * w * (sum({g: p for p, _, _, g in shares}.values()) + sum(n - p for p, n, _, _ in shares))
        pairs = h * sum(c * (n - c) + c * (c + 1) / 2.0 for _, n, c, _ in shares)
        return {"bytes": 2 * q + kv + q * 2 / w, "flops": 4.0 * w * pairs}
    if op == "weights":
        lens, h = _cache_lengths(case), case["heads"]
        rows, cells = float(sum(c for _, c in lens)), float(sum(n for n, _ in lens)) * hk
        pairs = h * sum(c * (n - c) + c * (c + 1) / 2.0 for n, c in lens)
        return {"bytes": rows * h * (2 * w + 4) + cells * (2 * w + 8), "flops": 2.0 * w * pairs}
    lens = _evict_lengths(case)
    kept = float(sum(min(n, case["keep"]) for n in lens)) * hk
    return {"bytes": 4.0 * sum(lens) * hk + kept * (8.0 * w + 4) + 4.0 * len(lens) * hk * case["keep"],
            "flops": float(sum(lens)) * hk}


# ------------------------------------------------------------------- the same in 64 bits, by definition


def _exact_packed(s):
    """Head by head: the quotient of sums, and its gradients by automatic differentiation in 64 bits."""
    case = s["case"]
    h, hk, w = case["heads"], case["kv_heads"], case["width"]
    q, k, v = (s[f].detach().double() for f in ("q", "k", "v"))
    y, dq, dk, dv = torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    lse = torch.zeros(h, case["rows"], dtype=torch.float64, device=DEV)
    starts = _starts(s["lens"])
    for a, e in zip(starts, starts[1:]):
        later = torch.ones(e - a, e - a, dtype=torch.bool, device=DEV).triu(1)
        for i in range(h):
            j = i // (h // hk)
            leaves = [t[a:e, x].clone().requires_grad_(case["step"]) for t, x in ((q, i), (k, j), (v, j))]
            logits = (leaves[0].mm(leaves[1].t()) / math.sqrt(w)).masked_fill(later, -math.inf)
            norm = torch.logsumexp(logits, 1)
            yi = torch.exp(logits - norm[:, None]).mm(leaves[2])
            y[a:e, i], lse[i, a:e] = yi.detach(), norm.detach()
            if case["step"]:
                grads = torch.autograd.grad(yi, leaves, s["dy"][a:e, i].double())
                dq[a:e, i] = grads[0]
                dk[a:e, j] += grads[1]
                dv[a:e, j] += grads[2]
    return (y, dq, dk, dv) if case["step"] else (y, lse)


def _exact_cached(s, use):
    """use(sequence, head, source head, logits [new tokens, positions], rows of the sequence, page and slot of its positions)."""
    case = s["case"]
    h, g, page = case["heads"], case["heads"] // case["kv_heads"], case["page"]
    q = s["q"].double()
    at = 0
    for b, (n, c) in enumerate(zip(s["lens"], s["counts"])):
        place = torch.arange(n, device=DEV)
        ids, slot = s["table"][b].long()[place // page], place % page
        seen = place[None, :] <= (n - c + torch.arange(c, device=DEV))[:, None]
        keys = s["k_pages"][ids, slot].double()
        for i in range(h):
            logits = q[at:at + c, i].mm(keys[:, i // g].t()) / math.sqrt(case["width"])
            use(b, i, i // g, torch.where(seen, logits, torch.full_like(logits, -math.inf)), slice(at, at + c), ids, slot)
        at += c


def _exact_prefix(s):
    y = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(s["q"].shape[1], s["q"].shape[0], dtype=torch.float64, device=DEV)

    def use(b, i, j, logits, rows, ids, slot):
        norm = torch.logsumexp(logits, 1)
        y[rows, i] = torch.exp(logits - norm[:, None]).mm(s["v_pages"][ids, slot, j].double())
        lse[i, rows] = norm

    _exact_cached(s, use)
    return y, lse


def _exact_weights(s):
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)

    def use(b, i, j, logits, rows, ids, slot):
        if i == j * (s["case"]["heads"] // s["case"]["kv_heads"]):  # the source head's first: what was there before
            old = s["lens"][b] - s["counts"][b]
            out[ids[:old], j, slot[:old]] = s["weights"][ids[:old], j, slot[:old]].double() * _DECAY
        out[ids, j, slot] += torch.exp(logits - s["lse"][i, rows].double()[:, None]).sum(0)

    _exact_cached(s, use)
    return out


def _exact_evict(s):
    """Sequence by sequence and head by head."""
    case = s["case"]
    page, keep = case["page"], case["keep"]
    outs = [torch.zeros(s[f].shape, dtype=torch.float64, device=DEV) for f in ("to_k", "to_v", "to_weights")]
    kept = torch.full((len(s["lens"]), case["kv_heads"], keep), -1, dtype=torch.int32, device=DEV)
    for b, n in enumerate(s["lens"]):
        place = torch.arange(n, device=DEV)
        ids, slot = s["table"][b].long()[place // page], place % page
        last = min(case["recent"], n)
        for j in range(case["kv_heads"]):
            weight = s["weights"][ids, j, slot].double()
            older = torch.sort(-weight[: n - last], stable=True).indices[: max(0, min(keep, n) - last)]
            stay = torch.cat([older.sort().values, place[n - last:]])
            to = torch.arange(stay.numel(), device=DEV)
            to_ids, to_slot = s["to_table"][b].long()[to // page], to % page
            outs[0][to_ids, to_slot, j] = s["k_pages"][ids[stay], slot[stay], j].double()
            outs[1][to_ids, to_slot, j] = s["v_pages"][ids[stay], slot[stay], j].double()
            outs[2][to_ids, j, to_slot] = weight[stay]
            kept[b, j, : stay.numel()] = stay.to(torch.int32)
    return (*outs, _ints([min(n, keep) for n in s["lens"]]), kept)


def exact(case, seed):
    s = prepare(case, seed)
    return dict(packed=_exact_packed, prefix=_exact_prefix, weights=_exact_weights, evict=_exact_evict)[case["op"]](s)
