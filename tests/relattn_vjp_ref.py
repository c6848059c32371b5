"""The cross attention VJP of given y and lse in 64 bits, with bounds that follow the roundings themselves.

What the kernels take is what they are given (y and lse as the forward wrote them), so neither's own error enters.  u is
the unit roundoff of the 16-bit type.  Two kinds of error:
  - of fp32, taken at its worst (terms added): of a weight ep = 2 (D + 8) 2^-24 scale sum_d |q_d k_d| + 2^-22 (|s| + |lse|)
    + 2^-20 (as in relattn_ref, and lse's product with log2 e), in binary16 2^-18 (an exponent of at most 64 is added to
    lse before it is rounded); of <dy, v> and <dy, y> D 2^-24 of the absolute terms; of
    sums over n (n / 16 + 64) 2^-24 of the absolute terms;
  - of the weights' and ds' roundings to the type: half a step each, u of the value, independent of each other, so the
    sum of b_j e_j is off by at most t sqrt(sum (b_j u)^2) but for a chance of 2 exp(-t^2 / 2) (Hoeffding), t = 8: 3e-14.
    In binary16 a rounding is off by at least half a smallest step: 2^-25 of the operand as it is scaled, so that the
    largest possible one (1 for p, 2 max_j |<dy_i, v_j>| <= 2 |dy_i|_1 max|v| for ds) is at least 2^13: 2^-38 of that.
    The largest |dy_i|_1 of all rows counts for dk.
  - an output is rounded once: u of it, in binary16 at least 2^-25.  From half a step below the type's next power of two
    on (65520 in binary16) that rounding gives an infinity of its sign, for want of a larger number.
"""
import torch

from tests.relattn_ref import U, sums

T = 8.0


def vjp(q, k, v, y, lse, dy, scale, dt, few, peak=None):
    """One head, float64: q, y, dy [n, D], k, v [m, D], lse [n].  few: delta is sum_j p dp instead of <dy, y>.  peak: the
    largest |dy_i|_1 of the rows that share the source head.  Returns (dq, dk, dv) and for each (worst, independent)."""
    u, D = U[dt], q.shape[1]
    n, m = q.shape[0], k.shape[0]
    half = dt == torch.float16
    s = q @ k.t() * scale
    ep = (2 * (D + 8) * 2.0 ** -24 * scale * (q.abs() @ k.abs().t()) + 2.0 ** -22 * (s.abs() + lse.abs()[:, None])
          + (2.0 ** -18 if half else 2.0 ** -20))
    p = torch.exp(s - lse[:, None])
    dp = dy @ v.t()
    dpe = D * 2.0 ** -24 * (dy.abs() @ v.abs().t())
    if few:
        delta = (p * dp).sum(1, keepdim=True)
        dle = (p * (ep * dp.abs() + dpe)).sum(1, keepdim=True) + sums(m) * (p * dp.abs()).sum(1, keepdim=True)
    else:
        delta = (dy * y).sum(1, keepdim=True)
        dle = D * 2.0 ** -24 * (dy * y).abs().sum(1, keepdim=True)
    ds = p * (dp - delta)
    lin = p * (dpe + dle) + (ep + 2.0 ** -22) * ds.abs()
    l1 = dy.abs().sum(1, keepdim=True)
    vmax = v.abs().max() if m else torch.zeros((), dtype=torch.float64)
    top = l1.max() if peak is None else peak
    rq = u * ds.abs() + (2.0 ** -38 * 2 * l1 * vmax if half else 0.0)
    rk = u * ds.abs() + (2.0 ** -38 * 2 * top * vmax if half else 0.0)
    rp = u * p + (2.0 ** -38 if half else 0.0)
    sq = lambda t: t * t
    dq, dk, dv = ds @ k * scale, ds.t() @ q * scale, p.t() @ dy
    wq = scale * (lin @ k.abs() + sums(m) * (ds.abs() @ k.abs()))
    wk = scale * (lin.t() @ q.abs() + sums(n) * (ds.abs().t() @ q.abs()))
    wv = (ep * p).t() @ dy.abs() + sums(n) * (p.t() @ dy.abs())
    return (dq, dk, dv), ((wq, sq(scale) * (sq(rq) @ sq(k))), (wk, sq(scale) * (sq(rk).t() @ sq(q))), (wv, sq(rp).t() @ sq(dy)))


def check(got, q, k, v, y, lse, dy, scale, tile, lens=None, what=""):
    """got: dq, dk, dv of a batch [B, H, N, D] over [B, Hk, S, D]; tile: sources up to which delta comes from the weights."""
    dt = q.dtype
    qd, kd, vd, yd, dyd, ld = (t.detach().double().cpu() for t in (q, k, v, y, dy, lse))
    B, H, N, D = q.shape
    Hk, S = k.shape[1], k.shape[2]
    G = H // Hk
    for b in range(B):
        n = S if lens is None else max(0, min(S, int(lens[b])))
        for j in range(Hk):
            heads = range(j * G, (j + 1) * G)
            peak = max(float(dyd[b, h].abs().sum(1).max()) for h in heads)
            sk = sv = 0.0
            ek, ev = [0.0, 0.0], [0.0, 0.0]
            for h in heads:
                (dq, dk, dv), (bq, bk, bv) = vjp(qd[b, h], kd[b, j, :n], vd[b, j, :n], yd[b, h], ld[b, h], dyd[b, h], scale, dt,
                                                 n <= tile, peak)
                within(got["dq"][b, h], dq, bq, dt, f"{what} dq {b, h}")
                sk, sv = sk + dk, sv + dv
                ek, ev = [x + e for x, e in zip(ek, bk)], [x + e for x, e in zip(ev, bv)]
            within(got["dk"][b, j, :n], sk, ek, dt, f"{what} dk {b, j}")
            within(got["dv"][b, j, :n], sv, ev, dt, f"{what} dv {b, j}")


def within(got, ref, bound, dt, what):
    err = (got.detach().double().cpu() - ref).abs()
    b = bound[0] + T * bound[1] ** 0.5
    b = b + U[dt] * (ref.abs() + b) + (2.0 ** -25 if dt == torch.float16 else 0.0)
    got = got.detach().double().cpu()
    past = (ref.abs() + b >= torch.finfo(dt).max) & (got == torch.sign(ref) * torch.inf)
    bad = ~((err <= b) | past)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} exceed the bound, the worst {float((err / b).nan_to_num(nan=1e30).max()):.3g} times"
