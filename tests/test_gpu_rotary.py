"""Rotary positions and the cache append against 64 bits.

An angle is formed in 64 bits and reduced there; sine and cosine of the rest (at most an eighth of a turn) are fp32
with 2 ulp and the reduction's rounding to fp32, 2^-24 of at most pi / 4: at most 4 * 2^-24 absolute.  The rotated
element is two products and a sum, amplitudes included: off by at most amp (|a| + |b|) 8 * 2^-24, then rounded once.
"""
import pytest
import torch

from tests.paged_ref import Batch

pytestmark = pytest.mark.gpu

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
U = {F16: 2.0 ** -11, BF16: 2.0 ** -8, F32: 2.0 ** -24}


def turned(x, pos, freq, amp, interleaved, sign=1.0):
    """x [..., heads, rows, width] float64, pos [..., rows]; the result and its bound (without the last rounding)."""
    rot = 2 * freq.numel()
    t = (pos.double()[..., None] * freq)[..., None, :, :]
    c, s = torch.cos(t) * amp, torch.sin(t) * amp * sign
    y, e = x.clone(), torch.zeros_like(x)
    if interleaved:
        i0, i1 = torch.arange(0, rot, 2), torch.arange(1, rot, 2)
    else:
        i0, i1 = torch.arange(rot // 2), torch.arange(rot // 2, rot)
    a, b = x[..., i0], x[..., i1]
    y[..., i0], y[..., i1] = a * c - b * s, a * s + b * c
    e[..., i0] = e[..., i1] = (a.abs() + b.abs()) * abs(amp) * 8 * 2.0 ** -24
    return y, e


def within(got, ref, e, dt, what):
    tiny = 2.0 ** -25 if dt == F16 else 0.0
    err = (got.double().cpu() - ref).abs()
    bad = ~(err <= e + U[dt] * (ref.abs() + e) + tiny)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()}, worst {err[bad].max()}"


CASES = [  # batch, heads, rows, width, rot, interleaved, type, amplitude, far
    (1, 1, 1, 64, 64, False, F16, 1.0, 1), (2, 3, 17, 128, 128, False, BF16, 1.0, 5000),
    (1, 4, 33, 128, 64, True, F16, 1.25, 1_000_000), (2, 2, 5, 80, 20, True, BF16, 1.0, 100),
    (3, 1, 7, 80, 80, False, F32, 0.5, 2 ** 31 - 1), (1, 5, 9, 37, 10, False, F32, 1.0, 1000),
    (1, 2, 300, 64, 16, False, BF16, 1.0, 30000), (1, 1, 3, 2, 2, True, F16, 1.0, 77), (1, 2, 4, 33, 32, True, F32, -1.0, 50),
    (4, 40, 65, 128, 128, True, BF16, 1.0, 4096), (2, 64, 2, 128, 32, False, F16, 1.0, 4096), (1, 3, 2, 12, 6, False, F16, 1.0, 9),
]


def setup(lib, B, H, N, D, rot, il, dt, amp, far, seed=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(B, H, N, D, generator=g).to(dt).cuda()
    pos = torch.randint(0, far, (B, N), generator=g, dtype=torch.int32)
    freq = lib.tiga_rotary_frequencies(rot)
    return x, pos, freq, lib.Rotary(freq.cuda(), il, amp)


@pytest.mark.parametrize("B,H,N,D,rot,il,dt,amp,far", CASES)
def test_against_64_bits(lib, B, H, N, D, rot, il, dt, amp, far):
    x, pos, freq, r = setup(lib, B, H, N, D, rot, il, dt, amp, far)
    y = lib.tiga_mp_rotary_fwd(x, pos.cuda(), r)
    dx = lib.tiga_mp_rotary_bwd(x, pos.cuda(), r)
    torch.cuda.synchronize()
    for got, sign in ((y, 1.0), (dx, -1.0)):
        ref, e = turned(x.double().cpu(), pos, freq, amp, il, sign)
        within(got, ref, e, dt, f"sign {sign}")
        assert torch.equal(got[..., rot:], x[..., rot:])


def test_layouts_positions_and_in_place(lib):
    x, pos, freq, r = setup(lib, 2, 4, 30, 64, 32, False, BF16, 1.0, 999)
    y = lib.tiga_mp_rotary_fwd(x, pos.cuda(), r)
    xn = x.permute(0, 2, 1, 3).contiguous()
    assert torch.equal(lib.tiga_mp_rotary_fwd(xn, pos.cuda(), r, layout="bnhd").permute(0, 2, 1, 3), y)
    assert torch.equal(lib.tiga_mp_rotary_fwd(x[0], pos[0].cuda(), r, layout="hnd"), y[0])
    one = lib.tiga_mp_rotary_fwd(x, pos[1].cuda(), r)             # one row of positions for the batch
    assert torch.equal(one[1], y[1]) and not torch.equal(one[0], y[0])
    z = x.clone()
    assert lib.tiga_mp_rotary_fwd(z, pos.cuda(), r, out=z) is z and torch.equal(z, y)
    ar = torch.arange(30, dtype=torch.int32, device="cuda")
    assert torch.equal(lib.tiga_mp_rotary_fwd(x, None, r), lib.tiga_mp_rotary_fwd(x, ar, r))
    # a part of a joint projection at an odd offset: rows that are not 16-byte aligned
    big = torch.randn(2, 30, 4, 71, generator=torch.Generator().manual_seed(1)).to(BF16).cuda()
    part = big[..., 3:67]
    got = lib.tiga_mp_rotary_fwd(part, pos.cuda(), r, layout="bnhd")
    assert torch.equal(got, lib.tiga_mp_rotary_fwd(part.contiguous(), pos.cuda(), r, layout="bnhd"))
    keep = big.clone()
    lib.tiga_mp_rotary_fwd(part, pos.cuda(), r, layout="bnhd", out=part)
    assert torch.equal(part, got) and torch.equal(big[..., :3], keep[..., :3]) and torch.equal(big[..., 67:], keep[..., 67:])


def test_gradient_is_the_adjoint_and_the_difference(lib):
    x, pos, freq, r = setup(lib, 1, 2, 12, 64, 64, True, F32, 1.1, 300)
    x.requires_grad_(True)
    dy = torch.randn(x.shape, generator=torch.Generator().manual_seed(2)).cuda()
    y = lib.rotary(x, pos.cuda(), r)
    y.backward(dy)
    # the map is linear: <dy, J d> by a difference of the 64-bit forward is exact
    d = torch.randn(x.shape, generator=torch.Generator().manual_seed(3), dtype=torch.float64)
    jd, e = turned(d, pos, freq, 1.1, True)
    lhs, rhs = (dy.double().cpu() * jd).sum(), (x.grad.double().cpu() * d).sum()
    scale = (dy.double().cpu().abs() * (d.abs() + 1)).sum() * 1.1 * 2
    assert abs(lhs - rhs) <= 12 * 2.0 ** -24 * scale
    lib.rotary(x, pos.cuda(), r).sum().backward()     # a cotangent of stride 0


def test_frequencies(lib):
    i = torch.arange(32, dtype=torch.float64)
    f = 10000.0 ** (-2 * i / 64)
    eq = lambda a, b: torch.allclose(a, b, rtol=1e-14, atol=0)
    assert eq(lib.tiga_rotary_frequencies(64), f)
    assert eq(lib.tiga_rotary_frequencies(64, scaling="linear", factor=4), f / 4)
    assert eq(lib.tiga_rotary_frequencies(64, scaling="base", factor=4), (10000.0 * 4 ** (64 / 62)) ** (-2 * i / 64))
    b = lib.tiga_rotary_frequencies(64, scaling="bands", factor=8, trained=8192, low=1, high=4)
    turns = 8192 * f / (2 * torch.pi)
    assert eq(b[turns >= 4], f[turns >= 4]) and eq(b[turns <= 1], f[turns <= 1] / 8)
    mid = (turns > 1) & (turns < 4)
    assert mid.any() and (b[mid] < f[mid]).all() and (b[mid] > f[mid] / 8).all()


@pytest.mark.parametrize("lens,H,Hk,D,page,dt,rot,il", [
    ([(1, 1)], 4, 1, 64, 16, F16, 64, False), ([(17, 1), (16, 1), (1, 1), (900, 1)], 8, 2, 128, 16, BF16, 128, True),
    ([(40, 33), (0, 0), (70, 7), (5, 5)], 6, 3, 64, 8, F16, 32, False), ([(300, 300), (129, 1)], 2, 2, 128, 64, BF16, 16, True),
    ([(20 + i, 1) for i in range(70)], 1, 1, 64, 1, BF16, 64, False), ([(9, 2)], 3, 1, 128, 4, F16, 2, True)])
@pytest.mark.parametrize("rows_first", [False, True])
def test_append(lib, lens, H, Hk, D, page, dt, rot, il, rows_first):
    bt = Batch(lens, Hk, D, page, dt, seed=5, rows_first=rows_first, tail=3)
    layout = "nhd" if rows_first else "hnd"
    k, v, q = (bt.tokens(n, rows_first) for n in (Hk, Hk, H))
    freq = lib.tiga_rotary_frequencies(rot)
    r = lib.Rotary(freq.cuda(), il, 1.0)
    k0, v0 = bt.k.clone(), bt.v.clone()
    hnd = (lambda t: t.permute(1, 0, 2)) if rows_first else (lambda t: t)
    q_out = torch.full_like(q, 9.0)
    lib.tiga_mp_cache_append(bt.cache(lib), k, v, bt.dst_ptr, r, q=q, layout=layout, q_out=q_out)
    torch.cuda.synchronize()
    assert (hnd(q_out)[:, bt.rows:] == 9.0).all()
    written = torch.zeros(bt.num_pages, page, dtype=torch.bool)
    for b, (n, c) in enumerate(lens):
        rows = slice(bt.ptr[b], bt.ptr[b] + c)
        pos = torch.arange(n - c, n)
        ids, slot = bt.table[b].cpu().long()[pos // page], pos % page
        written[ids, slot] = True
        ref, e = turned(hnd(k)[:, rows].double().cpu(), pos, freq, 1.0, il)
        within(bt.k[ids.cuda(), :, slot.cuda()].permute(1, 0, 2), ref, e, dt, "k")
        assert torch.equal(bt.v[ids.cuda(), :, slot.cuda()].permute(1, 0, 2), hnd(v)[:, rows])
        ref, e = turned(hnd(q)[:, rows].double().cpu(), pos, freq, 1.0, il)
        within(hnd(q_out)[:, rows], ref, e, dt, "q")
    keep = ~written[:, None, :, None].cuda()
    assert torch.equal(torch.where(keep, bt.k, 0 * k0), torch.where(keep, k0, 0 * k0))
    assert torch.equal(torch.where(keep, bt.v, 0 * v0), torch.where(keep, v0, 0 * v0))
    # without a rotation k is stored as it is; q may be rotated in place
    lib.tiga_mp_cache_append(bt.cache(lib), k, v, bt.dst_ptr, layout=layout)
    lib.tiga_mp_cache_append(bt.cache(lib), k, v, bt.dst_ptr, r, q=q, layout=layout, q_out=q)
    torch.cuda.synchronize()
    assert torch.equal(hnd(q)[:, :bt.rows], hnd(q_out)[:, :bt.rows])


def test_append_without_rotation(lib):
    bt = Batch([(30, 12), (5, 1)], 2, 64, 16, F16, seed=6)
    k, v = bt.tokens(2), bt.tokens(2)
    assert lib.tiga_mp_cache_append(bt.cache(lib), k, v, bt.dst_ptr) is None
    gk, gv = bt.gathered(0)
    assert torch.equal(gk[:, 18:], k[:, :12].cpu()) and torch.equal(gv[:, 18:], v[:, :12].cpu())


def test_append_to_bad_pages_stores_nothing_there(lib):
    bt = Batch([(30, 1), (40, 1), (50, 1), (3, 1), (20, 1)], 2, 64, 16, BF16, seed=7)
    k, v, q = bt.tokens(2), bt.tokens(2), bt.tokens(4)
    bt.table[0, 1] = bt.num_pages
    bt.table[1, 2] = -5
    bt.length[2] = 16 * bt.table.shape[1] + 1
    bt.length[3] = 0
    r = lib.Rotary(lib.tiga_rotary_frequencies(64).cuda())
    k0 = bt.k.clone()
    out = lib.tiga_mp_cache_append(bt.cache(lib), k, v, bt.dst_ptr, r, q=q)
    torch.cuda.synchronize()
    changed = (bt.k != k0).any(3).any(1).nonzero().tolist()
    assert changed == [[int(bt.table[4, 1]), 3]]
    assert torch.equal(out[:, 3], q[:, 3])                     # no position: copied
    assert not torch.equal(out[:, 0], q[:, 0])
    bt.dst_ptr.copy_(torch.tensor([3, 2, -9, 50, 1, 7], dtype=torch.int32))
    lib.tiga_mp_cache_append(bt.cache(lib), k, v, bt.dst_ptr, r, q=q)
    torch.cuda.synchronize()
