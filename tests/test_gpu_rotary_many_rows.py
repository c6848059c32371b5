"""Rotation and append of more rows than one grid of threads (2^32) counts."""
import pytest
import torch

pytestmark = pytest.mark.gpu

F16 = torch.float16


def turned(x, pos, freq):
    """Half-split pairs of the last axis, float64."""
    n = freq.numel()
    t = pos.double()[:, None] * freq
    y = x.double().clone()
    a, b = x[:, :n].double(), x[:, n:2 * n].double()
    y[:, :n], y[:, n:2 * n] = a * torch.cos(t) - b * torch.sin(t), a * torch.sin(t) + b * torch.cos(t)
    return y


def close(got, ref, what):
    # fp32 products of values below 2 and an angle of 4 units: 2^-20; rounded once: 2^-11 relative
    err = (got.double() - ref).abs()
    fits = bool((err <= 2.0 ** -11 * (ref.abs() + 2.0 ** -20) + 2.0 ** -20).all())
    assert fits, f"{what}: {err.max()}"


def test_rotation(lib):
    """2^31 rows of three elements: two threads a row."""
    rows = (1 << 31) + 77
    x = torch.empty(1, 1, rows, 3, dtype=F16, device="cuda")
    x.view(-1)[:] = 1.5
    x[..., 1] = -0.5
    freq = torch.tensor([0.37], dtype=torch.float64)
    rot = lib.Rotary(freq.cuda())
    spots = [torch.arange(s, s + 300, device="cuda").clamp_(max=rows - 1) for s in (0, 1 << 30, (1 << 31) - 150, rows - 300)]
    before = [x[0, 0, i].clone() for i in spots]
    lib.tiga_mp_rotary_fwd(x, None, rot, out=x)
    torch.cuda.synchronize()
    for i, b in zip(spots, before):
        close(x[0, 0, i], turned(b, i, freq.cuda()), f"rows from {int(i[0])}")
    whole = 0
    for part in x.view(-1, 3).split(1 << 27):                    # every row was turned: its length is kept, its angle is not
        whole += int(((part[:, 0].float() ** 2 + part[:, 1].float() ** 2 - 2.5).abs() < 0.01).sum())
    assert whole == rows


@pytest.mark.parametrize("rot", [20, 64])                        # element by element (a block a token), and in slots
def test_append(lib, rot):
    n, page, D = (1 << 24) + 5, 1 << 15, 64
    pages = -(-n // page)
    k = torch.empty(n, 1, D, dtype=F16, device="cuda")
    k[:] = torch.linspace(-1, 1, D, device="cuda").half()
    kp, vp = (torch.zeros(pages, 1, page, D, dtype=F16, device="cuda") for _ in range(2))
    table = torch.arange(pages, dtype=torch.int32, device="cuda")[None]
    cache = lib.KvCache(kp, vp, table, torch.tensor([n], dtype=torch.int32, device="cuda"))
    freq = lib.tiga_rotary_frequencies(rot)
    lib.tiga_mp_cache_append(cache, k, k, torch.tensor([0, n], dtype=torch.int32, device="cuda"), lib.Rotary(freq.cuda()),
                             layout="nhd")
    torch.cuda.synchronize()
    flat_k, flat_v = kp.view(-1, D), vp.view(-1, D)
    stored = torch.equal(flat_v[:n], k[:, 0]), bool((flat_v[n:] == 0).all()), bool((flat_k[n:] == 0).all())
    assert stored == (True, True, True)
    for s in (0, n // 2, (1 << 24) - 250, n - 200):
        i = torch.arange(s, s + 200, device="cuda")
        close(flat_k[i], turned(k[i, 0], i, freq.cuda()), f"tokens from {s}")
    empty = int((flat_k[:n, :rot // 2] == 0).all(1).sum())
    assert empty == 0
