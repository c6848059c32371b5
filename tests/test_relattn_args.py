"""Host-side checks of the rectangular-relation entry points: every call returns before anything reaches a device."""
import ctypes as C
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def b():
    from paper_2609_24802_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    binding.load()
    return binding


FAKE = 0x10000


def view(b, data=FAKE, batch=1 << 12, head=1 << 9, row=64):
    return b._View(data, batch, head, row)


def test_struct_layouts_match_the_header(tmp_path, b):
    import subprocess
    names = dict(tiga_view=b._View, tiga_cross=b._Cross, tiga_rotary=b._Rotary, tiga_cache=b._Cache)
    lines = "".join(
        f'  printf("%zu", sizeof({c}));\n' + "".join(f'  printf(" %zu", offsetof({c}, {f}));\n' for f, _ in s._fields_)
        + '  printf("\\n");\n' for c, s in names.items())
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "tiga_mp.h"\nint main(void) {\n' + lines + "  return 0;\n}\n")
    subprocess.check_call(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "l")])
    out = subprocess.check_output([str(tmp_path / "l")]).decode().strip().split("\n")
    for line, s in zip(out, names.values()):
        assert [int(x) for x in line.split()] == [C.sizeof(s)] + [getattr(s, f).offset for f, _ in s._fields_], s


CROSS = dict(num_dst=10, num_src=20, batch=2, heads=4, kv_heads=2, width=64, dtype=0, src_len=None)


@pytest.mark.parametrize("over,code", [
    (dict(num_dst=-1), -1), (dict(num_src=-1), -1), (dict(batch=-1), -1), (dict(heads=-4), -1), (dict(kv_heads=-2), -1),
    (dict(heads=5), -1), (dict(heads=4, kv_heads=0), -1), (dict(dtype=2), -1), (dict(dtype=9), -1), (dict(width=96), -3),
    (dict(width=32), -3), (dict(num_dst=1 << 31), -3), (dict(num_src=(1 << 31) - 1024), -3), (dict(src_len=0x10001), -1),
    (dict(batch=1 << 20, kv_heads=1, heads=1), -3), (dict(num_dst=1 << 30, heads=1024), -3)])
def test_cross_relation(b, over, code):
    L, rel = b.load(), b._Cross(**{**CROSS, **over})
    v = view(b)
    args = [C.byref(v)] * 3 + [0.125, C.byref(v), None, C.c_void_p(FAKE), 1 << 40, None]
    assert L.tiga_mp_attention_cross_fwd(C.byref(rel), *args) == code and L.tiga_last_error()
    assert L.tiga_mp_attention_cross_fwd_workspace(C.byref(rel)) == 0
    assert L.tiga_mp_attention_cross_bwd_workspace(C.byref(rel)) == 0
    args = [C.byref(v)] * 4 + [C.c_void_p(FAKE), C.byref(v), 0.125] + [C.byref(v)] * 3 + [C.c_void_p(FAKE), 1 << 40, None]
    assert L.tiga_mp_attention_cross_bwd(C.byref(rel), *args) == code


def test_cross_arguments(b):
    L, rel = b.load(), b._Cross(**CROSS)
    E, W = b.TIGA_EINVAL, b.TIGA_EWORKSPACE
    ok = view(b)

    def fwd(rel=rel, q=ok, k=ok, v=ok, scale=0.125, y=ok, lse=None, ws=FAKE, n=1 << 40):
        r = lambda x: C.byref(x) if x is not None else None
        return L.tiga_mp_attention_cross_fwd(r(rel), r(q), r(k), r(v), scale, r(y), lse, C.c_void_p(ws), n, None)

    assert fwd(rel=None) == E
    for name in ("q", "k", "v", "y"):
        for bad in (None, view(b, data=None), view(b, data=FAKE + 8), view(b, row=60), view(b, head=-64), view(b, batch=4)):
            assert fwd(**{name: bad}) == E, (name, bad)
    for bad in (view(b, row=0), view(b, head=0), view(b, batch=0)):
        assert fwd(y=bad) == E and b"overlap" in L.tiga_last_error()
    for s in (0.0, -1.0, float("inf"), float("nan")):
        assert fwd(scale=s) == E
    assert fwd(lse=C.c_void_p(FAKE + 2)) == E
    assert fwd(ws=0) == E and fwd(ws=FAKE + 16) == E and fwd(n=0) == W
    # nothing to compute: no tensors needed
    for over in (dict(batch=0), dict(heads=0, kv_heads=0), dict(num_dst=0)):
        assert fwd(rel=b._Cross(**{**CROSS, **over}), q=None, k=None, v=None, y=None, ws=0, n=0) == b.TIGA_OK

    def bwd(q=ok, k=ok, v=ok, y=ok, lse=FAKE, dy=ok, dq=ok, dk=ok, dv=ok, scale=0.125, ws=FAKE, n=1 << 40):
        r = lambda x: C.byref(x) if x is not None else None
        return L.tiga_mp_attention_cross_bwd(C.byref(rel), r(q), r(k), r(v), r(y), C.c_void_p(lse), r(dy), scale, r(dq),
                                             r(dk), r(dv), C.c_void_p(ws), n, None)

    for name in ("q", "k", "v", "y", "dy"):
        for bad in (None, view(b, data=FAKE + 8), view(b, row=60)):
            assert bwd(**{name: bad}) == E, name
    for name in ("dq", "dk", "dv"):
        assert bwd(**{name: view(b, row=0)}) == E and bwd(**{name: view(b, data=FAKE + 2)}) == E
    assert bwd(lse=0) == E and bwd(lse=FAKE + 1) == E and bwd(scale=float("nan")) == E
    assert bwd(ws=0) == E and bwd(n=0) == W


def cache(b, **over):
    v = view(b)
    d = dict(num_pages=8, page_size=16, kv_heads=2, width=64, dtype=0, batch=3, table_width=4, k=v, v=v, table=FAKE, length=FAKE)
    d.update(over)
    return b._Cache(**d)


@pytest.mark.parametrize("over,code", [
    (dict(num_pages=-1), -1), (dict(num_pages=0), -1), (dict(page_size=0), -1), (dict(page_size=24), -1),
    (dict(page_size=-16), -1), (dict(page_size=1 << 16), -3), (dict(kv_heads=-1), -1), (dict(width=96), -3),
    (dict(dtype=2), -1), (dict(batch=-1), -1), (dict(batch=1 << 16), -3), (dict(table_width=-1), -1),
    (dict(num_pages=1 << 31), -3), (dict(table_width=1 << 27), -3), (dict(table=None), -1), (dict(length=None), -1),
    (dict(table=FAKE + 2), -1), (dict(k=None), -1), (dict(v=None), -1), ("unaligned", -1), ("overlap", -1)])
def test_cache_checks(b, over, code):
    if over == "unaligned":
        over = dict(k=view(b, data=FAKE + 8))
    elif over == "overlap":
        over = dict(v=view(b, batch=0))
    over = {f: (b._View() if x is None and f in "kv" else x) for f, x in over.items()}
    L, c, v, p = b.load(), cache(b, **over), view(b), C.c_void_p(FAKE)
    r = C.byref
    assert L.tiga_mp_attention_paged_fwd(r(c), 5, p, 4, r(v), 0.125, r(v), None, p, 1 << 40, None) == code
    assert L.tiga_mp_cache_append(r(c), 5, p, r(v), r(v), None, 0, None, None, None) == code
    assert L.tiga_cache_validate(r(c), 5, p, None) == code


def test_paged_and_append_arguments(b):
    L, c, v, p, r = b.load(), cache(b), view(b), C.c_void_p(FAKE), C.byref
    E = b.TIGA_EINVAL
    rot = b._Rotary(FAKE, 64, 0, 1.0)

    def fwd(c=c, n=5, ptr=p, heads=4, q=v, scale=0.125, y=v, lse=None, ws=p, nb=1 << 40):
        o = lambda x: r(x) if x is not None else None
        return L.tiga_mp_attention_paged_fwd(o(c), n, ptr, heads, o(q), scale, o(y), lse, ws, nb, None)

    assert fwd(c=None) == E and fwd(n=-1) == E and fwd(ptr=None) == E and fwd(heads=3) == E and fwd(heads=-2) == E
    assert fwd(q=None) == E and fwd(y=None) == E and fwd(q=view(b, row=4)) == E and fwd(y=view(b, head=0)) == E
    assert fwd(scale=0.0) == E and fwd(ws=None) == E and fwd(nb=0) == b.TIGA_EWORKSPACE
    assert fwd(n=1 << 30) == b.TIGA_EUNSUPPORTED and fwd(lse=C.c_void_p(FAKE + 1)) == E
    assert fwd(n=0, q=None, y=None) == b.TIGA_OK and fwd(c=cache(b, batch=0), q=None, y=None) == b.TIGA_OK
    assert L.tiga_mp_attention_paged_fwd_workspace(r(c), 5, 4) > 0
    assert L.tiga_mp_attention_paged_fwd_workspace(r(c), 5, 3) == 0

    def app(c=c, n=5, ptr=p, k=v, v=v, rot=rot, heads=4, q=v, qo=v):
        o = lambda x: r(x) if x is not None else None
        return L.tiga_mp_cache_append(o(c), n, ptr, o(k), o(v), o(rot), heads, o(q), o(qo), None)

    assert app(c=None) == E and app(n=-1) == E and app(ptr=None) == E and app(k=None) == E and app(v=None) == E
    assert app(rot=None) == E                                   # q without a rotation
    assert app(qo=None) == E and app(qo=view(b, row=128)) == E   # in place with other strides
    assert app(heads=-1) == E and app(n=1 << 30, heads=8) == b.TIGA_EUNSUPPORTED
    assert app(n=0, k=None, v=None, q=None) == b.TIGA_OK
    for bad in (b._Rotary(None, 64, 0, 1.0), b._Rotary(FAKE, 66, 0, 1.0), b._Rotary(FAKE, 7, 0, 1.0), b._Rotary(FAKE, 0, 0, 1.0),
                b._Rotary(FAKE, 64, 2, 1.0), b._Rotary(FAKE, 64, 0, float("nan")), b._Rotary(FAKE + 4, 64, 0, 1.0)):
        assert app(rot=bad) == E


def test_rotary_arguments(b):
    L, r = b.load(), C.byref
    E = b.TIGA_EINVAL
    ok, rot = view(b), b._Rotary(FAKE, 64, 0, 1.0)
    for name in ("tiga_mp_rotary_fwd", "tiga_mp_rotary_bwd"):
        def call(batch=2, heads=3, rows=4, width=64, dt=0, x=ok, pos=None, pb=0, rot=rot, y=ok):
            o = lambda t: r(t) if t is not None else None
            return getattr(L, name)(batch, heads, rows, width, dt, o(x), pos, pb, o(rot), o(y), None)

        assert call(batch=-1) == E and call(heads=-1) == E and call(rows=-1) == E and call(width=0) == E and call(dt=3) == E
        assert call(width=1 << 16) == b.TIGA_EUNSUPPORTED and call(rows=1 << 39) == b.TIGA_EUNSUPPORTED
        assert call(x=None) == E and call(y=None) == E and call(x=view(b, data=FAKE + 1)) == E
        assert call(dt=2, y=view(b, data=FAKE + 2)) == E and call(x=view(b, row=-64)) == E and call(pb=-1) == E
        assert call(y=view(b, head=0, data=FAKE * 2)) == E and call(y=view(b, row=128)) == E
        assert call(pos=C.c_void_p(FAKE + 2)) == E and call(rot=None) == E and call(rot=b._Rotary(FAKE, 66, 0, 1.0)) == E
        assert call(rows=0, x=None, y=None) == b.TIGA_OK
    f = (C.c_double * 8)()
    freq = lambda rot=16, base=1e4, kind=0, factor=2.0, trained=100.0, low=1.0, high=4.0, out=f: L.tiga_rotary_frequencies(
        rot, base, kind, factor, trained, low, high, out)
    assert freq() == b.TIGA_OK and f[0] == 1.0
    assert freq(rot=15) == E and freq(rot=0) == E and freq(base=0.0) == E and freq(base=float("inf")) == E and freq(kind=4) == E
    assert freq(kind=1, factor=0.0) == E and freq(kind=2, rot=2) == E and freq(kind=3, low=4.0) == E and freq(out=None) == E
    assert freq(kind=3, trained=0.0) == E and freq(kind=1, factor=float("nan")) == E


def test_empty_caches(b):
    """Without sequences or heads nothing is read, so nothing is asked for; queries of no cache are refused."""
    L, r, none = b.load(), C.byref, b._View(None, 0, 0, 0)
    for over in (dict(batch=0), dict(kv_heads=0), dict(batch=0, num_pages=0)):
        c = cache(b, **{**over, "k": none, "v": none, "table": None, "length": None})
        assert L.tiga_cache_validate(r(c), 5, None, None) == b.TIGA_OK
        assert L.tiga_mp_cache_append(r(c), 5, None, None, None, None, 0, None, None, None) == b.TIGA_OK
    c, v, rot = cache(b, kv_heads=0), view(b), b._Rotary(FAKE, 64, 0, 1.0)
    assert L.tiga_mp_cache_append(r(c), 5, C.c_void_p(FAKE), r(v), r(v), r(rot), 4, r(v), r(v), None) == b.TIGA_EINVAL


def test_binding_refuses_host_tensors(b):
    import torch
    x = torch.zeros(1, 1, 4, 64, dtype=torch.float16)
    with pytest.raises(TypeError):
        b.tiga_mp_attention_cross_fwd(x, x, x)
    with pytest.raises(TypeError):
        b.Rotary(torch.zeros(4, dtype=torch.float64))
    with pytest.raises(TypeError):
        b.KvCache(x, x, torch.zeros(1, 1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32))
    with pytest.raises(ValueError):
        b.tiga_rotary_frequencies(8, scaling="other")


def test_a_workspace_holds_every_smaller_problem(b):
    """Growing any size of a problem never shrinks its workspace."""
    L, r = b.load(), C.byref
    grow = [1, 2, 3, 5, 16, 17, 31, 64, 65, 100, 128, 129, 256, 257, 500, 512, 513, 1024, 4096, 20_000, 200_000]
    base = dict(num_dst=40, num_src=700, batch=3, heads=8, kv_heads=4, width=128, dtype=0, src_len=None)
    for width in (64, 128):
        for query in (L.tiga_mp_attention_cross_fwd_workspace, L.tiga_mp_attention_cross_bwd_workspace):
            for other in (dict(), dict(num_dst=1), dict(num_src=50), dict(num_dst=3000, batch=1)):
                for f in ("num_dst", "num_src", "batch"):
                    sizes = [query(r(b._Cross(**{**base, "width": width, **other, f: n}))) for n in grow]
                    assert min(sizes) >= 256 and sizes == sorted(sizes), (f, other, sizes)
                kv = [query(r(b._Cross(**{**base, "width": width, **other, "heads": 2 * n, "kv_heads": n}))) for n in grow[:15]]
                assert kv == sorted(kv)
    for over in (dict(), dict(page_size=2), dict(kv_heads=1), dict(table_width=400)):
        for group in (1, 8, 32):
            size = lambda n, **o: L.tiga_mp_attention_paged_fwd_workspace(
                r(c := cache(b, **{**over, **o})), n, c.kv_heads * group)
            for seq in ([size(n) for n in grow], [size(17, batch=n) for n in grow if n < 1 << 16],
                        [size(300, batch=n) for n in grow if n < 1 << 16], [size(9, table_width=n) for n in grow],
                        [size(100, table_width=n) for n in grow], [size(30, kv_heads=n) for n in grow[:15]]):
                assert min(seq) >= 256 and seq == sorted(seq), (over, group, seq)
