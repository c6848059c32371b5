"""What the rotation's backward needs is guarded against changes in place between forward and backward."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("changed", ["freq", "pos"])
def test_a_change_in_place_is_noticed(lib, changed):
    freq = lib.tiga_rotary_frequencies(64).cuda()
    rot, pos = lib.Rotary(freq), torch.arange(5, dtype=torch.int32, device="cuda")
    x = torch.randn(1, 2, 5, 64, device="cuda", requires_grad=True)
    lib.rotary(x, pos, rot).sum().backward()                      # unchanged: fine
    y = lib.rotary(x, pos, rot)
    (freq if changed == "freq" else pos).mul_(2)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
    lib.rotary(x, pos, rot).sum().backward()                      # a new forward takes the new values


def test_without_positions(lib):
    rot = lib.Rotary(lib.tiga_rotary_frequencies(64).cuda())
    x = torch.randn(1, 2, 5, 64, device="cuda", requires_grad=True)
    lib.rotary(x, None, rot).backward(x.detach())
    assert torch.equal(x.grad, lib.tiga_mp_rotary_bwd(x.detach(), None, rot))
