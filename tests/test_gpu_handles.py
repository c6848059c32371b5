"""KvCache and Rotary hold their tensors' addresses: contents change freely, tensors are not replaced unnoticed."""
import pytest
import torch

from tests.paged_ref import Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["k_pages", "v_pages", "table", "length"])
def test_a_cache_keeps_its_tensors(lib, name):
    cache = Batch([(30, 1), (20, 1)], 2, 64, 16, torch.float16).cache(lib)
    t = getattr(cache, name)
    with pytest.raises(AttributeError, match="cannot be replaced"):
        setattr(cache, name, t.clone())
    assert getattr(cache, name) is t
    setattr(cache, name, t)


def test_lengths_grow_in_place(lib):
    bt = Batch([(31, 1), (20, 1)], 2, 64, 16, torch.float16)
    cache, q = bt.cache(lib), bt.tokens(4)
    cache.length -= 2                                      # an in-place operation and the same tensor again
    y = lib.tiga_mp_attention_paged_fwd(cache, q, bt.dst_ptr)
    other = lib.KvCache(bt.k, bt.v, bt.table, torch.tensor([29, 18], dtype=torch.int32, device="cuda"))
    assert torch.equal(y, lib.tiga_mp_attention_paged_fwd(other, q, bt.dst_ptr))


def test_a_rotation_keeps_its_frequencies(lib):
    rot = lib.Rotary(lib.tiga_rotary_frequencies(64).cuda())
    with pytest.raises(AttributeError, match="cannot be replaced"):
        rot.freq = rot.freq / 2
    x = torch.randn(1, 1, 4, 64, device="cuda")
    rot.freq /= 2
    half = lib.Rotary(lib.tiga_rotary_frequencies(64).cuda() / 2)
    assert torch.equal(lib.tiga_mp_rotary_fwd(x, None, rot), lib.tiga_mp_rotary_fwd(x, None, half))
