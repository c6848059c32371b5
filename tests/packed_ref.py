"""Causal attention of packed sequences in 64 bits on the CPU, with what each output may be off by (relattn_ref)."""
import torch

from tests import relattn_ref as R


class Packed:
    """Random packed sequences on the GPU: q, dy [H, N, D], k, v [Hk, N, D] ("hnd"); `lead` and `tail` rows of no sequence."""

    def __init__(self, lens, H, Hk, D, dt, seed=0, lead=0, tail=0):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.H, self.Hk, self.D, self.dt = list(lens), H, Hk, D, dt
        self.ptr = [lead]
        for n in lens:
            self.ptr.append(self.ptr[-1] + n)
        self.N = self.ptr[-1] + tail
        make = lambda h: torch.randn(h, self.N, D, generator=g).to(dt).cuda()
        self.q, self.k, self.v, self.dy = make(H), make(Hk), make(Hk), make(H)
        self.ptr_t = torch.tensor(self.ptr, dtype=torch.int32, device="cuda")

    def outside(self):
        keep = torch.zeros(self.N, dtype=torch.bool)
        keep[self.ptr[0]:self.ptr[-1]] = True
        return ~keep


def reference(s, scale, gradients=True):
    """Outputs and bounds; rows of no sequence: y, gradients 0 and lse -inf, exactly."""
    H, Hk, N, D, dt = s.H, s.Hk, s.N, s.D, s.dt
    q, k, v, dy = (t.detach().double().cpu() for t in (s.q, s.k, s.v, s.dy))
    z = lambda *a: torch.zeros(*a, dtype=torch.float64)
    out = dict(y=z(H, N, D), lse=torch.full((H, N), -torch.inf, dtype=torch.float64), dq=z(H, N, D), dk=z(Hk, N, D),
               dv=z(Hk, N, D))
    bound = {n: torch.zeros_like(t) for n, t in out.items()}
    for a, e in zip(s.ptr, s.ptr[1:]):
        if a == e:
            continue
        here = slice(a, e)
        seen = torch.ones(e - a, e - a, dtype=torch.bool).tril()
        for h in range(H):
            j = h // (H // Hk)
            f = R.rows(q[h, here], k[j, here], v[j, here], seen, scale)
            out["y"][h, here], out["lse"][h, here] = f["y"], f["lse"]
            bound["y"][h, here], bound["lse"][h, here] = f["y_bound"](dt), f["lse_bound"]
            if gradients:
                g, b, _ = R.grads(f, q[h, here], k[j, here], v[j, here], dy[h, here], scale, dt)
                out["dq"][h, here], bound["dq"][h, here] = g[0], b[0]
                for n, x, y in (("dk", g[1], b[1]), ("dv", g[2], b[2])):
                    out[n][j, here] += x
                    bound[n][j, here] += y
        for n in ("dk", "dv"):
            bound[n][:, here] += R.U[dt] * out[n][:, here].abs() + (2.0 ** -25 if dt == torch.float16 else 0.0)
    return out, bound


def check(lib, s, what, scale=None, gradients=True, ref=None):
    y, lse = lib.tiga_mp_attention_packed_fwd(s.q, s.k, s.v, s.ptr_t, scale, want_lse=True)
    torch.cuda.synchronize()
    out, bound = ref or reference(s, s.D ** -0.5 if scale is None else scale, gradients)
    R.assert_within(lse, out["lse"], bound["lse"], what + " lse")
    R.assert_within(y, out["y"], bound["y"], what + " y")
    if gradients:
        g = lib.tiga_mp_attention_packed_bwd(s.q, s.k, s.v, y, lse, s.dy, s.ptr_t, scale)
        torch.cuda.synchronize()
        for n in ("dq", "dk", "dv"):
            R.assert_within(g[n], out[n], bound[n], f"{what} {n}")
    return y, lse
