"""Nothing is written behind a workspace of the size that the query tells, and results do not depend on what lies in it."""
import pytest
import torch

from tests.test_gpu_prefix_attention import Grouped

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16

# lengths (with the new tokens, new tokens), groups (sequences, shared), heads, source heads, width, page, type, rows behind
CASES = [
    ([(5, 1)], [], 1, 1, 64, 16, F16, 0),
    ([(300, 1), (290, 1), (40, 0)], [(2, 256)], 4, 2, 64, 16, F16, 3),
    ([(4000, 1), (4500, 1), (3900, 2)], [(3, 3840)], 16, 2, 128, 16, BF16, 0),
    ([(600, 90), (640, 100)], [(2, 500)], 8, 1, 128, 64, F16, 200),
    ([(1000 + i, 1) for i in range(70)], [(30, 900), (40, 700)], 4, 4, 64, 32, BF16, 0),
    ([(0, 0), (0, 0)], [(2, 0)], 4, 4, 128, 16, BF16, 9),
    ([(9000, 1), (33000, 20)], [(1, 50), (1, 0)], 4, 1, 64, 64, F16, 0),
    ([(2300, 2100), (150, 1)], [(2, 128)], 4, 2, 64, 8, BF16, 0),
]


@pytest.mark.parametrize("lens,groups,H,Hk,D,page,dt,tail", CASES)
def test_guarded(lib, lens, groups, H, Hk, D, page, dt, tail):
    bt = Grouped(lens, groups, Hk, D, page, dt, seed=51, tail=tail, copies=True)
    cache, q, L, C = bt.cache(lib), bt.tokens(H), lib.load(), lib.C
    weights = torch.rand(bt.num_pages, Hk, page, generator=bt.g).cuda()
    keep = max(1, min(n for n, _ in lens) // 2)

    def both(call, size):
        """The call with a workspace of its own, of zeros and of ones, and what lies behind the latter two."""
        outs = [call(None)]
        for fill in (0, 0xff):
            whole = torch.full((size + (1 << 20),), fill, dtype=torch.uint8, device="cuda")
            outs.append(call(whole[:size]))
            torch.cuda.synchronize()
            assert (whole[size:] == fill).all()
        for a, b, c in zip(*outs):
            a, b, c = (t[:, :bt.rows] if t.shape[:2] == (H, bt.num_dst) else t for t in (a, b, c))
            assert torch.equal(a, b) and torch.equal(a, c)
        return outs[0]

    prefix = lib._prefix(cache, bt.group_ptr, bt.group_len)
    y, lse = both(lambda ws: lib.tiga_mp_attention_prefix_fwd(cache, q, bt.dst_ptr, bt.group_ptr, bt.group_len, want_lse=True, ws=ws),
                  L.tiga_mp_attention_prefix_fwd_workspace(cache.ref, C.byref(prefix), bt.num_dst, H))
    both(lambda ws: (lib.tiga_mp_cache_weights(cache, q, lse, bt.dst_ptr, weights, out=weights.clone(), ws=ws),),
         L.tiga_mp_cache_weights_workspace(cache.ref, bt.num_dst, H))
    state = [t.clone() for t in (bt.k, bt.v, bt.length, weights)]

    def evict(ws):
        for t, old in zip((bt.k, bt.v, bt.length, weights), state):
            t.copy_(old)
        kept = lib.tiga_mp_cache_evict(cache, weights, keep=keep, recent=keep // 2, ws=ws)
        return kept, bt.k.clone(), bt.v.clone(), bt.length.clone(), weights.clone()

    both(evict, L.tiga_mp_cache_evict_workspace(cache.ref, cache.ref, keep))
