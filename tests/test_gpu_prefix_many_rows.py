"""Attention behind shared prefixes with as many rows as make the join's threads more than one grid of them counts (2^32)."""
import pytest
import torch

from tests import relattn_ref as R

pytestmark = pytest.mark.gpu

F16 = torch.float16


def test_every_row_is_written(lib):
    """512 prompts of 2048 tokens, 128 heads of width 128: 2^27 rows.  All have the same pages and queries, so the same results."""
    n, H, D, page, batch = 2048, 128, 128, 128, 512
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 200 << 30:
        pytest.skip("takes 180 GB of device memory")
    g = torch.Generator().manual_seed(71)
    k, v = (torch.randn(n // page, 1, page, D, generator=g).to(F16).cuda() for _ in range(2))
    ints = lambda t: t.to(torch.int32).cuda()
    table = ints(torch.arange(n // page).expand(batch, -1).contiguous())
    one = torch.randn(1, 1, D, generator=g).to(F16)
    q = one.cuda().expand(H, batch * n, D)
    y = torch.full((H, batch * n, D), float("nan"), dtype=F16, device="cuda")
    call = lambda b, q, y: lib.tiga_mp_attention_prefix_fwd(
        lib.KvCache(k, v, table[:b], ints(torch.full((b,), n))), q, ints(torch.arange(b + 1) * n), ints(torch.tensor([0, b])),
        ints(torch.tensor([0])), y=y)
    call(batch, q, y)
    torch.cuda.synchronize()
    first = y[:, :n]
    f = R.rows(one[0].double().expand(n, D), *(t.double().cpu().reshape(n, D) for t in (k, v)),
               torch.ones(n, n, dtype=torch.bool).tril(), D ** -0.5)
    for h in (0, 77, H - 1):
        R.assert_within(first[h], f["y"], f["y_bound"](F16), f"head {h}")
    for b in range(1, batch):
        assert torch.equal(y[:, b * n:(b + 1) * n], first), b
    del q, y, first
    torch.cuda.empty_cache()
