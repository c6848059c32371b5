"""Workspaces that a caller hands over are looked at before anything is launched."""
import pytest
import torch

from tests.paged_ref import Batch

pytestmark = pytest.mark.gpu


def calls(lib):
    q = torch.randn(1, 2, 5, 64, device="cuda").half()
    k = torch.randn(1, 2, 700, 64, device="cuda").half()
    y, lse = lib.tiga_mp_attention_cross_fwd(q, k, k, want_lse=True)
    bt = Batch([(300, 1), (200, 1)], 2, 64, 16, torch.float16)
    qp = bt.tokens(4)
    return [lambda ws: lib.tiga_mp_attention_cross_fwd(q, k, k, ws=ws),
            lambda ws: lib.tiga_mp_attention_cross_bwd(q, k, k, y, lse, y, ws=ws)["dk"],
            lambda ws: lib.tiga_mp_attention_paged_fwd(bt.cache(lib), qp, bt.dst_ptr, ws=ws)]


@pytest.mark.parametrize("i", range(3))
def test_given_workspaces(lib, i):
    call = calls(lib)[i]
    n = 64 << 20
    for bad in (torch.empty(n, dtype=torch.uint8), bytearray(n)):
        with pytest.raises(TypeError):
            call(bad)
    with pytest.raises(ValueError):
        call(torch.empty(1, dtype=torch.uint8, device="cuda").expand(n))
    with pytest.raises(lib.TigaError) as e:
        call(torch.empty(256, dtype=torch.uint8, device="cuda"))
    assert e.value.code == lib.TIGA_EWORKSPACE
    ref = call(None)
    for ws in (torch.empty(n, dtype=torch.uint8, device="cuda"), torch.empty(n // 4, dtype=torch.float32, device="cuda")):
        assert torch.equal(call(ws), ref)
