"""The append's rows outside every sequence: those before dst_ptr[0] have no position, those behind the last are left alone."""
import pytest
import torch

from tests.paged_ref import Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rot", [64, 20])            # in 16-byte slots, element by element
@pytest.mark.parametrize("lens", [[(30, 3), (9, 1)], [(40, 20), (0, 0), (50, 17)], [(2000, 1500), (7, 7)]])
def test_rows_before_the_first_sequence(lib, lens, rot):
    bt = Batch(lens, 2, 64, 16, torch.bfloat16, seed=1, tail=4)
    lead = 5
    k, v, q = bt.tokens(2), bt.tokens(2), bt.tokens(4)
    r = lib.Rotary(lib.tiga_rotary_frequencies(rot).cuda())
    pages = bt.k.clone(), bt.v.clone()
    ref = lib.tiga_mp_cache_append(bt.cache(lib), k, v, bt.dst_ptr, r, q=q, q_out=torch.full_like(q, 9.0))
    want = bt.k.clone(), bt.v.clone()
    bt.k.copy_(pages[0]), bt.v.copy_(pages[1])
    front = lambda t: torch.cat([torch.randn(t.shape[0], lead, 64, device="cuda").to(t.dtype), t], 1)
    kl, vl, ql = front(k), front(v), front(q)
    out = torch.full_like(ql, 9.0)
    lib.tiga_mp_cache_append(bt.cache(lib), kl, vl, bt.dst_ptr + lead, r, q=ql, q_out=out)
    torch.cuda.synchronize()
    assert torch.equal(out[:, :lead], ql[:, :lead])                         # copied, unrotated
    assert torch.equal(out[:, lead:], ref)                                  # 9 behind the last sequence
    assert torch.equal(bt.k, want[0]) and torch.equal(bt.v, want[1])        # and nothing of them stored
    lib.tiga_mp_cache_append(bt.cache(lib), kl, vl, bt.dst_ptr + lead, r, q=ql, q_out=ql)
    torch.cuda.synchronize()
    assert torch.equal(ql[:, :lead + bt.rows], out[:, :lead + bt.rows])     # in place


@pytest.mark.parametrize("lens", [[(30, 1), (9, 1)], [(300, 200), (50, 1)]])
def test_attention_leaves_them(lib, lens):
    bt = Batch(lens, 2, 64, 16, torch.float16, seed=2, tail=3)
    q = bt.tokens(4)
    ref = lib.tiga_mp_attention_paged_fwd(bt.cache(lib), q, bt.dst_ptr)
    ql = torch.cat([q[:, :2], q], 1)
    y = torch.full_like(ql, 3.0)
    lib.tiga_mp_attention_paged_fwd(bt.cache(lib), ql, bt.dst_ptr + 2, y=y)
    torch.cuda.synchronize()
    assert (y[:, :2] == 3.0).all() and (y[:, 2 + bt.rows:] == 3.0).all()
    assert torch.equal(y[:, 2:2 + bt.rows], ref[:, :bt.rows])
