"""Attention over other relations than the square ones, and what feeds it, as measurable cases.

Four operators: cross attention (destinations and sources of different counts, padded batches, heads
that share sources; a forward, and a training step with the gradients of q, k and v), attention of new
tokens over a paged cache (prompt chunks and single tokens), rotary positions (forward and gradient),
and the append of new keys and values to the cache's pages with the rotation on the way.

With ``own`` false a pass is elementary torch operations in 32 bits (angles in 64), rounded once; with
``own`` true it is the calls of ``paper_2609_24802_amd.binding``.  ``exact`` is the definition in 64 bits.
"""
import math
import random

import torch

own = False

DEV = "cuda:0"


def listed():
    return [
        # generation with an encoder-decoder model: one new token a sequence over ragged encoder states
        dict(name="cross_token", op="cross", batch=16, heads=16, kv_heads=16, num_dst=1, num_src=1500, width=64,
             dtype="f16", ragged=True, step=False),
        # training of image tokens that read a short text: few sources, many destinations
        dict(name="cross_short_step", op="cross", batch=4, heads=8, kv_heads=8, num_dst=4096, num_src=77, width=64,
             dtype="bf16", ragged=False, step=True),
        # training of a decoder over padded encoder states, one of them empty
        dict(name="cross_ragged_step", op="cross", batch=8, heads=16, kv_heads=16, num_dst=449, num_src=1500, width=64,
             dtype="f16", ragged=True, step=True),
        # training of a reader over a long document, four heads to a source head; the largest
        dict(name="cross_long_step", op="cross", batch=2, heads=16, kv_heads=4, num_dst=2048, num_src=8192, width=128,
             dtype="bf16", ragged=False, step=True),
        # one user's next token: latency
        dict(name="paged_token_1", op="paged", batch=1, heads=32, kv_heads=8, width=128, page=16, longest=4001,
             chunk=1, chunks=0, dtype="bf16"),
        # a serving batch's next tokens, lengths between a few and thousands
        dict(name="paged_token_64", op="paged", batch=64, heads=32, kv_heads=8, width=128, page=16, longest=8192,
             chunk=1, chunks=0, dtype="bf16"),
        # next tokens over long contexts
        dict(name="paged_token_long", op="paged", batch=4, heads=16, kv_heads=2, width=128, page=64, longest=131072,
             chunk=1, chunks=0, dtype="f16"),
        # a chunk of a long prompt beside the next tokens of other users
        dict(name="paged_chunk_mixed", op="paged", batch=17, heads=16, kv_heads=4, width=128, page=32, longest=16001,
             chunk=1023, chunks=1, dtype="bf16"),
        # training: queries and keys of four sequences turned by their positions, and the gradient turned back
        dict(name="rotary_step", op="rotary", batch=4, heads=40, rows=4096, width=128, rot=128, interleaved=False,
             scaling="none", far=0, dtype="bf16", step=True),
        # serving: a quarter of the width, adjacent pairs, positions far out under stretched frequencies
        dict(name="rotary_part_far", op="rotary", batch=1, heads=36, rows=61, width=64, rot=16, interleaved=True,
             scaling="bands", far=1_000_000, dtype="f16", step=False),
        # next tokens of a serving batch: keys turned and stored, queries turned
        dict(name="append_token_64", op="append", batch=64, heads=32, kv_heads=8, width=128, page=16, longest=500,
             chunk=1, chunks=0, rot=128, interleaved=False, dtype="bf16"),
        # prompt chunks entering the cache
        dict(name="append_chunks", op="append", batch=5, heads=16, kv_heads=4, width=128, page=64, longest=9000,
             chunk=2047, chunks=4, rot=64, interleaved=True, dtype="f16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["cross", "cross", "cross", "paged", "paged", "paged", "rotary", "append"])
    dtype, width = rng.choice(["f16", "bf16"]), rng.choice([64, 128])
    if op == "rotary":
        case = dict(op=op, batch=rng.randint(1, 8), heads=_log(rng, 1, 64), rows=_log(rng, 1, 4096),
                    width=rng.choice([64, 80, 128]), interleaved=rng.random() < 0.5,
                    scaling=rng.choice(["none", "linear", "base", "bands"]), far=rng.choice([0, 0, 30_000, 1_000_000]),
                    dtype=rng.choice(["f16", "bf16", "f32"]), step=rng.random() < 0.5)
        case["rot"] = rng.choice([case["width"], case["width"], case["width"] // 2, case["width"] // 4])
        while case["batch"] * case["heads"] * case["rows"] * case["width"] > 4 * 40 * 4096 * 128:
            case["rows"] = max(1, case["rows"] // 2)
        return case
    kv_heads, group = _log(rng, 1, 16), rng.choice([1, 1, 2, 4, 8])
    if op == "cross":
        case = dict(op=op, batch=_log(rng, 1, 16), heads=kv_heads * group, kv_heads=kv_heads,
                    num_dst=rng.choice([1, _log(rng, 1, 4096), _log(rng, 1, 4096)]), num_src=_log(rng, 1, 8192),
                    width=width, dtype=dtype, ragged=rng.random() < 0.5, step=rng.random() < 0.6)
        while case["batch"] * case["heads"] * case["num_dst"] * case["num_src"] * width > 2 * 16 * 2048 * 8192 * 128:
            big = max(("batch", "num_dst", "num_src"), key=lambda f: case[f])
            case[big] = max(1, case[big] // 2)
        return case
    case = dict(op=op, batch=_log(rng, 1, 64), heads=kv_heads * group, kv_heads=kv_heads, width=width,
                page=rng.choice([16, 32, 64, 128]), longest=_log(rng, 20, 65536), chunk=1, chunks=0, dtype=dtype)
    if rng.random() < 0.5 or op == "append":
        case["chunk"] = _log(rng, 1, min(2048, case["longest"]))
        case["chunks"] = rng.randint(1, min(4, case["batch"]))
    cells = 4 * 131072 * 2 * 128 if op == "paged" else 5 * 9000 * 4 * 128
    while case["batch"] * case["longest"] * kv_heads * width > cells:
        big = max(("batch", "longest"), key=lambda f: case[f] / (64 if f == "longest" else 1))
        case[big] = max(1, case[big] // 2)
    case["chunk"] = min(case["chunk"], case["longest"])
    case["chunks"] = min(case["chunks"], case["batch"])
    while case["chunks"] * case["chunk"] * case["longest"] * case["heads"] * width > 1023 * 16001 * 16 * 128:
        case["chunk"] = max(1, case["chunk"] // 2)
    if op == "append":
        case["rot"], case["interleaved"] = rng.choice([width, width, width // 2]), rng.random() < 0.5
    return case


# ------------------------------------------------------------------------------------- inputs

_TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def _src_lengths(case):
    """Sources of each sequence of a cross attention batch: the longest whole, one empty where the batch is large."""
    n, b = case["num_src"], case["batch"]
    if not case["ragged"]:
        return [n] * b
    rng = random.Random(b * 1_000_003 + n)
    lens = [n] + [rng.randint((n + 2) // 3, n) for _ in range(b - 1)]
    if b > 4:
        lens[b // 2] = 0
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


def _frequencies(rot, scaling):
    """Radians a position of each pair, fp64 [rot / 2], and the amplitude."""
    i = torch.arange(rot // 2, dtype=torch.float64)
    factor, base = 8.0, 10000.0
    if scaling == "base":
        base *= factor ** (rot / (rot - 2)) if rot > 2 else 1.0
    f = base ** (-2.0 * i / rot)
    if scaling == "linear":
        f = f / factor
    if scaling == "bands":  # slow pairs, under one turn over 8192 positions, stretched; fast ones, over 4, kept
        turns = 8192.0 * f / (2.0 * math.pi)
        keep = ((turns - 1.0) / 3.0).clamp(0.0, 1.0)
        f = f * (keep + (1.0 - keep) / factor)
        return f.to(DEV), 0.1 * math.log(factor) + 1.0
    return f.to(DEV), 1.0


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed) * 7919 + 29)
    dt = _TYPES[case["dtype"]]
    randn = lambda *s: torch.randn(*s, generator=g, device=DEV).to(dt)
    ints = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)
    op, width = case["op"], case["width"]
    s = dict(case=case)
    if op == "cross":
        b, h, hk, nd, ns = (case[f] for f in ("batch", "heads", "kv_heads", "num_dst", "num_src"))
        # the projections' own layout: rows of all heads, keys and values side by side
        s["q"] = randn(b, nd, h, width)
        kv = randn(b, ns, 2, hk, width)
        s["k"], s["v"] = kv[:, :, 0], kv[:, :, 1]
        s["len"] = ints(_src_lengths(case)) if case["ragged"] else None
        if case["step"]:
            s["dy"] = randn(b, nd, h, width)
        if own and case["step"]:
            s["q"].requires_grad_(True)
            s["k"], s["v"] = s["k"].detach().requires_grad_(True), s["v"].detach().requires_grad_(True)
        return s
    if op == "rotary":
        s["freq"], s["amp"] = _frequencies(case["rot"], case["scaling"])
        shape = (case["batch"], case["rows"], case["heads"], width)
        s["x"] = randn(*shape)
        s["pos"] = torch.arange(case["rows"], device=DEV, dtype=torch.int32).expand(case["batch"], -1).contiguous()
        if case["far"]:
            s["pos"] = torch.randint(0, case["far"], shape[:2], generator=g, device=DEV, dtype=torch.int32)
        if case["step"]:
            s["dy"] = randn(*shape)
        if own:
            from paper_2609_24802_amd import binding as tb
            s["rotary"] = tb.Rotary(s["freq"], interleaved=case["interleaved"], amplitude=s["amp"])
            s["x"].requires_grad_(case["step"])
        return s
    lens = _cache_lengths(case)
    page, hk = case["page"], case["kv_heads"]
    need = [-(-n // page) for n, _ in lens]
    pages = sum(need) + 3
    order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    table = torch.full((len(lens), max(need)), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, c in enumerate(need):
        table[b, :c] = order[at:at + c]
        at += c
    s["k_pages"], s["v_pages"] = randn(pages, page, hk, width), randn(pages, page, hk, width)
    s["table"], s["length"] = table, ints([n for n, _ in lens])
    ptr = [0]
    for _, c in lens:
        ptr.append(ptr[-1] + c)
    s["lens"], s["ptr"] = lens, ints(ptr)
    s["q"] = randn(ptr[-1], case["heads"], width)
    if op == "append":
        s["freq"], s["amp"] = _frequencies(case["rot"], "none")
        s["k"], s["v"] = randn(ptr[-1], hk, width), randn(ptr[-1], hk, width)
    if own:
        from paper_2609_24802_amd import binding as tb
        s["cache"] = tb.KvCache(s["k_pages"].permute(0, 2, 1, 3), s["v_pages"].permute(0, 2, 1, 3), table, s["length"])
        if op == "append":
            s["rotary"] = tb.Rotary(s["freq"], interleaved=case["interleaved"], amplitude=s["amp"])
    return s


# ------------------------------------------------------------------------------ plain passes, 32 bits


def _plain_cross(s):
    case = s["case"]
    b, h, hk, nd, ns, w = (case[f] for f in ("batch", "heads", "kv_heads", "num_dst", "num_src", "width"))
    scale, g = w ** -0.5, h // hk
    # [batch, source head, group rows, width]: the heads of a group are further rows over the same sources
    rows = lambda t: t.float().view(b, nd, hk, g, w).permute(0, 2, 3, 1, 4).reshape(b, hk, g * nd, w)
    back = lambda t: t.view(b, hk, g, nd, w).permute(0, 3, 1, 2, 4).reshape(b, nd, h, w)
    q = rows(s["q"])
    k, v = (s[f].float().permute(0, 2, 1, 3).contiguous() for f in ("k", "v"))
    kt = k.transpose(2, 3).contiguous()
    sc = torch.matmul(q, kt) * scale
    if s["len"] is not None:
        off = torch.arange(ns, device=DEV)[None, :] >= s["len"][:, None]
        sc.masked_fill_(off[:, None, None, :], -math.inf)
    top = sc.amax(-1, keepdim=True).clamp_(min=-3e38)
    p = sc.sub_(top).exp_()
    mass = p.sum(-1, keepdim=True)
    p /= torch.where(mass > 0, mass, torch.ones_like(mass))
    y = torch.matmul(p, v)
    dt = s["q"].dtype
    if not case["step"]:
        lse = (mass.log() + top).masked_fill_(mass == 0, -math.inf)
        return back(y).to(dt), lse.view(b, h, nd)
    dy = rows(s["dy"])
    dv = torch.matmul(p.transpose(2, 3).contiguous(), dy)
    ds = torch.matmul(dy, v.transpose(2, 3).contiguous())
    ds -= (dy * y).sum(-1, keepdim=True)
    ds *= p
    dq = torch.matmul(ds, k) * scale
    dk = torch.matmul(ds.transpose(2, 3).contiguous(), q) * scale
    return back(y).to(dt), back(dq).to(dt), dk.permute(0, 2, 1, 3).to(dt), dv.permute(0, 2, 1, 3).to(dt)


def _plain_paged(s):
    case = s["case"]
    hk, w, page = case["kv_heads"], case["width"], case["page"]
    h, g = case["heads"], case["heads"] // case["kv_heads"]
    dt = s["q"].dtype
    y = torch.empty_like(s["q"])
    lse = torch.empty(h, s["q"].shape[0], device=DEV)
    at = 0
    for b, (n, c) in enumerate(s["lens"]):
        ids = s["table"][b, : -(-n // page)].long()
        k = s["k_pages"][ids].view(-1, hk, w)[:n].permute(1, 2, 0).float().contiguous()
        v = s["v_pages"][ids].view(-1, hk, w)[:n].permute(1, 0, 2).float().contiguous()
        q = s["q"][at:at + c].float().view(c, hk, g, w).permute(1, 2, 0, 3).reshape(hk, g * c, w)
        sc = (torch.matmul(q, k) * w ** -0.5).view(hk, g, c, n)
        if c > 1:
            late = torch.arange(n, device=DEV)[None, :] > torch.arange(n - c, n, device=DEV)[:, None]
            sc.masked_fill_(late, -math.inf)
        top = sc.amax(-1, keepdim=True)
        p = sc.sub_(top).exp_()
        mass = p.sum(-1, keepdim=True)
        o = torch.matmul(p.view(hk, g * c, n), v).view(hk, g, c, w) / mass
        y[at:at + c] = o.permute(2, 0, 1, 3).reshape(c, h, w).to(dt)
        lse[:, at:at + c] = (mass.log() + top).view(h, c)
        at += c
    return y, lse


def _plain_turn(x, pos, freq, amp, interleaved, back=False):
    """x [..., heads, width] in fp32, the first 2 * len(freq) of the width turned by pos [...] * freq."""
    rot = 2 * freq.numel()
    angle = pos.double()[..., None, None] * freq
    c, s = (angle.cos() * amp).float(), (angle.sin() * (-amp if back else amp)).float()
    x = x.float()
    out = x.clone()
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        out[..., 0:rot:2], out[..., 1:rot:2] = a * c - b * s, a * s + b * c
    else:
        a, b = x[..., : rot // 2], x[..., rot // 2:rot]
        out[..., : rot // 2], out[..., rot // 2:rot] = a * c - b * s, a * s + b * c
    return out


def _plain_append(s):
    case = s["case"]
    page = case["page"]
    count = s["ptr"][1:] - s["ptr"][:-1]
    rows = s["q"].shape[0]
    seq = torch.repeat_interleave(torch.arange(len(s["lens"]), device=DEV), count.long(), output_size=rows)
    pos = torch.arange(rows, device=DEV) - s["ptr"][seq] + s["length"][seq] - count[seq]
    ids, slot = s["table"][seq, pos // page].long(), pos % page
    turn = lambda t: _plain_turn(t, pos, s["freq"], s["amp"], case["interleaved"]).to(t.dtype)
    s["k_pages"][ids, slot] = turn(s["k"])
    s["v_pages"][ids, slot] = s["v"]
    return turn(s["q"]), s["k_pages"], s["v_pages"]


# -------------------------------------------------------------------------------------- passes


def _own(s):
    from paper_2609_24802_amd import binding as tb
    case = s["case"]
    op = case["op"]
    if op == "cross":
        if not case["step"]:
            return tb.tiga_mp_attention_cross_fwd(s["q"], s["k"], s["v"], s["len"], want_lse=True, layout="bnhd")
        y = tb.cross_attention(s["q"], s["k"], s["v"], s["len"], layout="bnhd")
        return (y,) + torch.autograd.grad(y, (s["q"], s["k"], s["v"]), s["dy"])
    if op == "paged":
        return tb.tiga_mp_attention_paged_fwd(s["cache"], s["q"], s["ptr"], want_lse=True, layout="nhd")
    if op == "rotary":
        if not case["step"]:
            return tb.tiga_mp_rotary_fwd(s["x"], s["pos"], s["rotary"], layout="bnhd")
        y = tb.rotary(s["x"], s["pos"], s["rotary"], layout="bnhd")
        return (y,) + torch.autograd.grad(y, (s["x"],), s["dy"])
    q = tb.tiga_mp_cache_append(s["cache"], s["k"], s["v"], s["ptr"], s["rotary"], q=s["q"], layout="nhd")
    return q, s["k_pages"], s["v_pages"]


def run(s):
    if own:
        return _own(s)
    case = s["case"]
    op = case["op"]
    if op == "cross":
        return _plain_cross(s)
    if op == "paged":
        return _plain_paged(s)
    if op == "rotary":
        y = _plain_turn(s["x"], s["pos"], s["freq"], s["amp"], case["interleaved"]).to(s["x"].dtype)
        if not case["step"]:
            return y
        return y, _plain_turn(s["dy"], s["pos"], s["freq"], s["amp"], case["interleaved"], True).to(s["x"].dtype)
    return _plain_append(s)


def work(case):
    op, w = case["op"], case["width"]
    size = 4.0 if case["dtype"] == "f32" else 2.0
    if op == "cross":
        b, h, hk, nd = (case[f] for f in ("batch", "heads", "kv_heads", "num_dst"))
        sources = sum(_src_lengths(case))
        q, kv, pairs = b * nd * h * w * size, 2.0 * sources * hk * w * size, float(h) * nd * sources
        if not case["step"]:
            return {"bytes": 2 * q + kv + 4.0 * b * h * nd, "flops": 4.0 * w * pairs}
        # q, k, v, dy in; y, dq, dk, dv out (whole, the padding's zeros among them)
        return {"bytes": 4 * q + kv + 2.0 * b * case["num_src"] * hk * w * size, "flops": 14.0 * w * pairs}
    if op == "rotary":
        x = float(case["batch"]) * case["rows"] * case["heads"]
        return {"bytes": 2.0 * x * w * size * (2 if case["step"] else 1),
                "flops": 3.0 * x * case["rot"] * (2 if case["step"] else 1)}
    lens = _cache_lengths(case)
    new = float(sum(c for _, c in lens))
    q = new * case["heads"] * w * size
    if op == "paged":
        kv = 2.0 * sum(n for n, _ in lens) * case["kv_heads"] * w * size
        pairs = sum(c * (n - c) + c * (c + 1) / 2.0 for n, c in lens)
        return {"bytes": 2 * q + kv + 4.0 * new * case["heads"], "flops": 4.0 * w * case["heads"] * pairs}
    return {"bytes": 2 * q + 4.0 * new * case["kv_heads"] * w * size,
            "flops": 3.0 * new * (case["heads"] + case["kv_heads"]) * case["rot"]}


# ------------------------------------------------------------------- the same in 64 bits, by definition


def _exact_cross(s):
    """Head by head: the quotient of sums, and its gradients by automatic differentiation in 64 bits."""
    case = s["case"]
    h, hk, nd, w = (case[f] for f in ("heads", "kv_heads", "num_dst", "width"))
    q, k, v = (s[f].detach().double() for f in ("q", "k", "v"))
    y = torch.zeros_like(q)
    lse = torch.full((case["batch"], h, nd), -math.inf, dtype=torch.float64, device=DEV)
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for b, n in enumerate(_src_lengths(case)):
        if n == 0:
            continue
        for i in range(h):
            j = i // (h // hk)
            qi, kj, vj = q[b, :, i].clone(), k[b, :n, j].clone(), v[b, :n, j].clone()
            if case["step"]:
                for t in (qi, kj, vj):
                    t.requires_grad_(True)
            logits = qi.mm(kj.t()) / math.sqrt(w)
            norm = torch.logsumexp(logits, 1)
            yi = torch.exp(logits - norm[:, None]).mm(vj)
            y[b, :, i], lse[b, i] = yi.detach(), norm.detach()
            if case["step"]:
                grads = torch.autograd.grad(yi, (qi, kj, vj), s["dy"][b, :, i].double())
                dq[b, :, i] = grads[0]
                dk[b, :n, j] += grads[1]
                dv[b, :n, j] += grads[2]
    return (y, dq, dk, dv) if case["step"] else (y, lse)


def _exact_paged(s):
    case = s["case"]
    h, g, page = case["heads"], case["heads"] // case["kv_heads"], case["page"]
    q = s["q"].double()
    y = torch.zeros_like(q)
    lse = torch.zeros(h, q.shape[0], dtype=torch.float64, device=DEV)
    at = 0
    for b, (n, c) in enumerate(s["lens"]):
        place = torch.arange(n, device=DEV)
        ids, slot = s["table"][b].long()[place // page], place % page
        for j in range(case["kv_heads"]):
            k, v = s["k_pages"][ids, slot, j].double(), s["v_pages"][ids, slot, j].double()
            for i in range(j * g, (j + 1) * g):
                logits = q[at:at + c, i].mm(k.t()) / math.sqrt(case["width"])
                seen = place[None, :] <= (n - c + torch.arange(c, device=DEV))[:, None]
                logits = torch.where(seen, logits, torch.full_like(logits, -math.inf))
                norm = torch.logsumexp(logits, 1)
                y[at:at + c, i] = torch.exp(logits - norm[:, None]).mm(v)
                lse[i, at:at + c] = norm
        at += c
    return y, lse


def _exact_turn(x, pos, freq, amp, interleaved):
    """Each pair as a complex number times amp e^(i pos freq)."""
    rot = 2 * freq.numel()
    x = x.detach().double()
    factor = torch.polar(torch.full((), amp, dtype=torch.float64, device=DEV).expand(pos.shape + freq.shape),
                         pos.double()[..., None] * freq)[..., None, :]
    head = x[..., :rot]
    if interleaved:
        z = torch.view_as_complex(head.reshape(head.shape[:-1] + (rot // 2, 2)).contiguous()) * factor
        turned = torch.view_as_real(z).reshape(head.shape)
    else:
        z = torch.complex(head[..., : rot // 2].contiguous(), head[..., rot // 2:].contiguous()) * factor
        turned = torch.cat([z.real, z.imag], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "cross":
        return _exact_cross(s)
    if op == "paged":
        return _exact_paged(s)
    if op == "rotary":
        y = _exact_turn(s["x"], s["pos"], s["freq"], s["amp"], case["interleaved"])
        if not case["step"]:
            return y
        return y, _exact_turn(s["dy"], s["pos"], -s["freq"], s["amp"], case["interleaved"])
    k_pages, v_pages = s["k_pages"].double(), s["v_pages"].double()
    q = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    at = 0
    for b, (n, c) in enumerate(s["lens"]):
        pos = torch.arange(n - c, n, device=DEV)
        ids, slot = s["table"][b].long()[pos // case["page"]], pos % case["page"]
        turn = lambda t: _exact_turn(t[at:at + c], pos, s["freq"], s["amp"], case["interleaved"])
        q[at:at + c] = turn(s["q"])
        k_pages[ids, slot], v_pages[ids, slot] = turn(s["k"]), s["v"][at:at + c].double()
        at += c
    return q, k_pages, v_pages
