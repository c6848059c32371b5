"""Source heads that no destination head reads: their gradients are 0, and written."""
import ctypes as C

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("S,D,dt", [(1, 64, torch.float16), (77, 128, torch.bfloat16), (1500, 64, torch.bfloat16)])
def test_gradients_without_heads(lib, S, D, dt):
    L, r = lib.load(), C.byref
    q = torch.empty(2, 0, 9, D, dtype=dt, device="cuda")
    k = torch.randn(2, 3, S, D, device="cuda").to(dt)
    dk, dv = torch.full_like(k, 7.0), torch.full_like(k, 7.0)
    rel, qv, kv, _, _ = lib._cross(q, k, k, None, "bhnd")
    view = lambda t: r(lib._rows(t, "t", lib._AXES["bhnd"])[1])
    ws = lib._workspace(L.tiga_mp_attention_cross_bwd_workspace(r(rel)), k.device)
    assert L.tiga_mp_attention_cross_bwd(r(rel), r(qv), r(kv), r(kv), r(qv), None, r(qv), 0.125, r(qv), view(dk), view(dv),
                                         lib._ptr(ws), ws.numel(), lib._stream()) == lib.TIGA_OK
    torch.cuda.synchronize()
    assert (dk == 0).all() and (dv == 0).all()
    y, lse = lib.tiga_mp_attention_cross_fwd(q, k, k, want_lse=True)
    g = lib.tiga_mp_attention_cross_bwd(q, k, k, y, lse, y)
    torch.cuda.synchronize()
    assert y.shape == q.shape and lse.shape == (2, 0, 9) and g["dq"].shape == q.shape
    assert (g["dk"] == 0).all() and (g["dv"] == 0).all()
