"""Attention over rectangular relations in 64 bits on the CPU, with what each output may be off by.

The bounds follow the arithmetic of the path (u is the unit roundoff of the 16-bit type):
  - scores: exact products, fp32 sums over the width D, one fp32 multiply by scale * log2(e), one exponential of
    2 ulp: a score is off by at most es = 2 (D + 8) 2^-24 scale sum_d |q_d k_d| + 2^-22 |s| + 2^-21, which is the
    relative error of its weight;
  - sums over n weights or terms: (n / 16 + 64) 2^-24 of the sum of the absolute terms (partial sums of at most
    16 parallel accumulators, joined);
  - a weight enters the value product rounded: u of it, and in binary16 at least 2^-25 (against a largest weight
    of at least 1);
  - every output is rounded once: u of its value.
"""
import torch

U = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


def sums(n):
    return (n / 16 + 64) * 2.0 ** -24


def rows(q, k, v, seen, scale):
    """One head: q [n, D], k and v [m, D] float64, seen bool [n, m].  Returns y, lse and what y and lse may be off by
    as functions of the type."""
    n, m = seen.shape
    D = q.shape[1]
    s = q @ k.t() * scale
    es = 2 * (D + 8) * 2.0 ** -24 * scale * (q.abs() @ k.abs().t()) + 2.0 ** -22 * s.abs() + 2.0 ** -21
    sm = s.masked_fill(~seen, -torch.inf)
    lse = torch.logsumexp(sm, 1) if m else torch.full((n,), -torch.inf, dtype=torch.float64)
    empty = lse == -torch.inf
    p = torch.exp(sm - torch.where(empty, torch.zeros_like(lse), lse)[:, None])
    y = p @ v
    yabs = p @ v.abs()
    worst = es.masked_fill(~seen, 0.0).amax(1, keepdim=True) if m else torch.zeros(n, 1, dtype=torch.float64)
    vmax = v.abs().max() if m else 0.0

    def y_bound(dt):
        u = U[dt]
        floor = m * 2.0 ** -25 * vmax + 2.0 ** -24 if dt == torch.float16 else 0.0
        return (2 * u + 2 * worst + 2 * sums(m)) * yabs + floor

    lse_bound = worst[:, 0] + sums(m) + 2.0 ** -21 * (1 + torch.where(empty, torch.zeros_like(lse), lse).abs())
    return dict(p=p, s=s, es=es, y=y, yabs=yabs, lse=lse, worst=worst, y_bound=y_bound, lse_bound=lse_bound)


def grads(f, q, k, v, dy, scale, dt):
    """The VJP of rows(...) = f for one head, and its bounds: (dq, dk, dv), (bounds).  The kernel takes delta from the
    forward's rounded y, so delta is off by at most sum_d |dy_d| (bound of y_d)."""
    u = U[dt]
    n, m = f["p"].shape
    D = q.shape[1]
    p = f["p"]
    dp = dy @ v.t()
    delta = (dy * f["y"]).sum(1, keepdim=True)
    ds = p * (dp - delta)
    dq, dk, dv = ds @ k * scale, ds.t() @ q * scale, p.t() @ dy
    ep = f["es"] + f["lse_bound"][:, None] + 2.0 ** -20            # relative error of a weight
    dpe = D * 2.0 ** -24 * (dy.abs() @ v.abs().t())                 # absolute error of <dy, v>
    dle = (dy.abs() * (f["y_bound"](dt) + D * 2.0 ** -24 * f["y"].abs())).sum(1, keepdim=True)
    half = dt == torch.float16
    pe = p * (u + ep) + (2.0 ** -25 if half else 0.0)
    dse = p * (dpe + dle) + (u + ep) * p * (dp.abs() + delta.abs()) + (2.0 ** -25 if half else 0.0)
    last = lambda t: u * t.abs() + (2.0 ** -25 if half else 0.0)
    bq = scale * (dse @ k.abs() + sums(m) * (ds.abs() @ k.abs())) + last(dq)
    bk = scale * (dse.t() @ q.abs() + sums(n) * (ds.abs().t() @ q.abs()))
    bv = pe.t() @ dy.abs() + sums(n) * (p.t() @ dy.abs())
    return (dq, dk, dv), (bq, bk, bv), last


def cross(q, k, v, lens, scale, dy=None):
    """Batch: q, dy [B, H, N, D], k, v [B, Hk, S, D] (any device, 16-bit).  Returns a dict of outputs and bounds."""
    dt = q.dtype
    B, H, N, D = q.shape
    Hk, S = k.shape[1], k.shape[2]
    q, k, v = (t.detach().double().cpu() for t in (q, k, v))
    dy = None if dy is None else dy.detach().double().cpu()
    z = lambda *s: torch.zeros(*s, dtype=torch.float64)
    out = dict(y=z(B, H, N, D), lse=z(B, H, N), dq=z(B, H, N, D), dk=z(B, Hk, S, D), dv=z(B, Hk, S, D))
    bound = {n: torch.zeros_like(t) for n, t in out.items()}
    for b in range(B):
        n = S if lens is None else max(0, min(S, int(lens[b])))
        for h in range(H):
            j = h // (H // Hk)
            f = rows(q[b, h], k[b, j, :n], v[b, j, :n], torch.ones(N, n, dtype=torch.bool), scale)
            out["y"][b, h], out["lse"][b, h] = f["y"], f["lse"]
            bound["y"][b, h], bound["lse"][b, h] = f["y_bound"](dt), f["lse_bound"]
            if dy is not None and n:
                g, e, last = grads(f, q[b, h], k[b, j, :n], v[b, j, :n], dy[b, h], scale, dt)
                out["dq"][b, h], bound["dq"][b, h] = g[0], e[0]
                out["dk"][b, j, :n] += g[1]
                out["dv"][b, j, :n] += g[2]
                bound["dk"][b, j, :n] += e[1]
                bound["dv"][b, j, :n] += e[2]
    if dy is not None:
        u = U[dt]
        for name in ("dk", "dv"):
            bound[name] += u * out[name].abs() + (2.0 ** -25 if dt == torch.float16 else 0.0)
            if lens is not None:   # the padding's gradients are exactly 0
                for b in range(B):
                    bound[name][b, :, max(0, min(S, int(lens[b]))):] = 0.0
    return out, bound


def assert_within(got, ref, bound, what):
    got = got.detach().double().cpu()
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    same = got == ref                                   # infinities that agree
    err = torch.where(same, torch.zeros_like(ref), (got - ref).abs())
    bad = ~(err <= bound)
    if bad.any():
        i = int(torch.where(bad, err - bound, torch.full_like(err, -1.0)).nan_to_num(nan=1e30).argmax())
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} exceed the bound; worst at flat {i}: got "
                             f"{got.flatten()[i]!r} ref {ref.flatten()[i]!r} bound {bound.flatten()[i]!r}")
