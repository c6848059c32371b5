"""The operators as a decoder uses them: keys and queries rotated and appended to the cache, causal attention over
the cache, then cross attention to an encoder's states; tokens fed one at a time, in chunks or all at once."""
import pytest
import torch

from tests import relattn_ref as R

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


class Layer:
    """Fixed inputs per token; the projections between the operators are left out."""

    def __init__(self, lib, B, H, Hk, D, total, enc, dt, page=16, seed=0):
        g = torch.Generator().manual_seed(seed)
        t = lambda *s: torch.randn(*s, generator=g).to(dt).cuda()
        self.lib, self.B, self.H, self.Hk, self.D, self.total, self.page = lib, B, H, Hk, D, total, page
        self.q, self.k, self.v = t(B, total, H, D), t(B, total, Hk, D), t(B, total, Hk, D)
        self.ek, self.ev = t(B, enc, Hk, D), t(B, enc, Hk, D)
        self.enc_len = torch.tensor([enc - 7 * b for b in range(B)], dtype=torch.int32, device="cuda")
        self.freq = lib.tiga_rotary_frequencies(D)
        self.rot = lib.Rotary(self.freq.cuda())
        per = -(-total // page)
        self.pages = torch.randperm(B * per, generator=g).to(torch.int32).view(B, per).cuda()
        self.dt, self.per = dt, per

    def feed(self, steps):
        """steps: new tokens of every sequence per call.  Returns the layer's rows [B, total, H, D] of both attentions."""
        lib, B = self.lib, self.B
        kp = torch.zeros(B * self.per, self.Hk, self.page, self.D, dtype=self.dt, device="cuda")
        vp = torch.zeros_like(kp)
        length = torch.zeros(B, dtype=torch.int32, device="cuda")
        cache = lib.KvCache(kp, vp, self.pages, length)
        own, cross = torch.empty_like(self.q), torch.empty_like(self.q)
        at = 0
        for c in steps:
            length += c
            ptr = torch.arange(0, B + 1, dtype=torch.int32, device="cuda") * c
            cut = lambda t: t[:, at:at + c].reshape(B * c, t.shape[2], self.D)
            q = lib.tiga_mp_cache_append(cache, cut(self.k), cut(self.v), ptr, self.rot, q=cut(self.q), layout="nhd")
            y = lib.tiga_mp_attention_paged_fwd(cache, q, ptr, layout="nhd").view(B, c, self.H, self.D)
            own[:, at:at + c] = y
            cross[:, at:at + c] = lib.tiga_mp_attention_cross_fwd(y, self.ek, self.ev, self.enc_len, layout="bnhd")
            at += c
        assert at == self.total
        return own, cross


@pytest.mark.parametrize("dt", [F16, BF16])
@pytest.mark.parametrize("H,Hk,D", [(4, 2, 64), (8, 1, 128)])
def test_chunks_and_single_tokens_agree_with_the_causal_attention(lib, H, Hk, D, dt):
    total = 75
    layer = Layer(lib, 3, H, Hk, D, total, 60, dt)
    # the square causal path on the same rotated rows, source heads repeated
    turn = lambda t: lib.tiga_mp_rotary_fwd(t, None, layer.rot, layout="bnhd")
    q, k = turn(layer.q), turn(layer.k)
    scale = D ** -0.5
    for steps in ([total], [1] * total, [40, 1, 1, 17, 16]):
        own, cross = layer.feed(steps)
        torch.cuda.synchronize()
        for b in range(3):
            for h in range(H):
                f = R.rows(q[b, :, h].double().cpu(), k[b, :, h * Hk // H].double().cpu(),
                           layer.v[b, :, h * Hk // H].double().cpu(), torch.ones(total, total).tril().bool(), scale)
                R.assert_within(own[b, :, h], f["y"], f["y_bound"](dt), f"own {len(steps)} calls")
        heads = lambda t: t.permute(0, 2, 1, 3)
        ref, bound = R.cross(heads(own), heads(layer.ek), heads(layer.ev), layer.enc_len, scale)
        R.assert_within(heads(cross), ref["y"], bound["y"], "cross")
        rep = lambda t: heads(t).repeat_interleave(H // Hk, 1)[0].contiguous()
        square = lib.tiga_mp_attention_fwd(heads(q)[0].contiguous(), rep(k), rep(layer.v))
        # both within their own distance of the exact rows; the square path forms its mass of rounded weights too
        f = [R.rows(q[0, :, h].double().cpu(), k[0, :, h * Hk // H].double().cpu(), layer.v[0, :, h * Hk // H].double().cpu(),
                    torch.ones(total, total).tril().bool(), scale) for h in range(H)]
        bound = torch.stack([x["y_bound"](dt) + (2 * R.U[dt] + 1e-4) * x["yabs"] for x in f]) + 2.0 ** -24
        if dt == F16:
            bound += total * 2.0 ** -25 * float(layer.v.abs().max())
        R.assert_within(square, heads(own)[0].double().cpu(), bound, "square")


def test_training_step_through_rotary_and_cross_attention(lib):
    """Gradients through both operators chained by autograd against 64 bits."""
    B, H, Hk, N, S, D, dt = 2, 4, 2, 40, 50, 64, F16
    g = torch.Generator().manual_seed(4)
    x = torch.randn(B, H, N, D, generator=g).to(dt).cuda().requires_grad_(True)
    k, v = (torch.randn(B, Hk, S, D, generator=g).to(dt).cuda().requires_grad_(True) for _ in range(2))
    dy = torch.randn(B, H, N, D, generator=g).to(dt).cuda()
    rot = lib.Rotary(lib.tiga_rotary_frequencies(D).cuda())
    q = lib.rotary(x, None, rot)
    q.retain_grad()
    y = lib.cross_attention(q, k, v)
    y.backward(dy)
    ref, bound = R.cross(q, k, v, None, D ** -0.5, dy)
    for t, name in ((q, "dq"), (k, "dk"), (v, "dv")):
        R.assert_within(t.grad, ref[name], bound[name], name)
    assert torch.equal(x.grad, lib.tiga_mp_rotary_bwd(q.grad, None, rot))


def test_generation_step_captured(lib):
    """Append, attention over the cache and cross attention in one graph; lengths advance between the replays."""
    B, H, Hk, D, page = 4, 8, 2, 128, 16
    g = torch.Generator().manual_seed(5)
    t = lambda *s: torch.randn(*s, generator=g).to(BF16).cuda()
    kp, vp = t(4 * 10, Hk, page, D), t(4 * 10, Hk, page, D)
    table = torch.randperm(40, generator=g).to(torch.int32).view(4, 10).cuda()
    length = torch.tensor([100, 1, 16, 47], dtype=torch.int32, device="cuda")
    ptr = torch.arange(5, dtype=torch.int32, device="cuda")
    q, k, v = t(B, H, D), t(B, Hk, D), t(B, Hk, D)
    ek, ev = t(B, Hk, 200, D), t(B, Hk, 200, D)
    enc = torch.tensor([200, 3, 0, 150], dtype=torch.int32, device="cuda")
    rot = lib.Rotary(lib.tiga_rotary_frequencies(D).cuda())

    def step(cache):
        qr = lib.tiga_mp_cache_append(cache, k, v, ptr, rot, q=q, layout="nhd")
        y = lib.tiga_mp_attention_paged_fwd(cache, qr, ptr, layout="nhd")
        return y, lib.tiga_mp_attention_cross_fwd(y.view(B, H, 1, D), ek, ev, enc)

    cache = lib.KvCache(kp, vp, table, length)
    kp2, vp2 = kp.clone(), vp.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(lib.KvCache(kp2, vp2, table, length))
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(cache)
    kp2.copy_(kp)
    vp2.copy_(vp)
    for i in range(5):
        for a in (q, k, v):
            a.copy_(torch.randn(a.shape, generator=g).to(BF16))
        graph.replay()
        ref = step(lib.KvCache(kp2, vp2, table, length))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, ref)), i
        assert torch.equal(kp, kp2) and torch.equal(vp, vp2)
        length += 1
