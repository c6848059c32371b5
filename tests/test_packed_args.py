"""Host-side checks of packed attention: every call returns before anything reaches a device."""
import ctypes as C
import os
import subprocess

import pytest
import torch

from tests.test_relattn_args import FAKE, ROOT, b, view  # noqa: F401

PACKED = dict(num_rows=100, batch=3, heads=4, kv_heads=2, width=64, dtype=0, ptr=FAKE)


def fwd(b, rel=None, q=0, k=0, v=0, scale=0.125, y=0, lse=None, ws=FAKE, n=1 << 40, **over):
    rel = b._Packed(**{**PACKED, **over}) if rel is None else rel
    r = lambda x: C.byref(view(b)) if x == 0 else C.byref(x) if x is not None else None
    return b.load().tiga_mp_attention_packed_fwd(C.byref(rel), r(q), r(k), r(v), scale, r(y), lse, C.c_void_p(ws), n, None)


def bwd(b, lse=FAKE, ws=FAKE, n=1 << 40, scale=0.125, over=None, **views):
    rel = b._Packed(**{**PACKED, **(over or {})})
    g = lambda name: C.byref(views[name]) if views.get(name, 0) not in (0, None) else None if name in views else C.byref(view(b))
    return b.load().tiga_mp_attention_packed_bwd(C.byref(rel), g("q"), g("k"), g("v"), g("y"), C.c_void_p(lse), g("dy"), scale,
                                                 g("dq"), g("dk"), g("dv"), C.c_void_p(ws), n, None)


def test_struct_layout_matches_the_header(tmp_path, b):  # noqa: F811
    s = b._Packed
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "tiga_mp.h"\nint main(void) {\n  printf("%zu", sizeof(tiga_packed));\n'
                   + "".join(f'  printf(" %zu", offsetof(tiga_packed, {f}));\n' for f, _ in s._fields_) + "  return 0;\n}\n")
    subprocess.check_call(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "l")])
    got = [int(x) for x in subprocess.check_output([str(tmp_path / "l")]).split()]
    assert got == [C.sizeof(s)] + [getattr(s, f).offset for f, _ in s._fields_]


@pytest.mark.parametrize("over,code", [
    (dict(num_rows=-1), -1), (dict(batch=-1), -1), (dict(heads=-4), -1), (dict(heads=5), -1), (dict(kv_heads=0), -1),
    (dict(dtype=2), -1), (dict(width=96), -3), (dict(num_rows=1 << 31), -3), (dict(num_rows=1 << 30), -3),
    (dict(batch=1 << 20), -3), (dict(ptr=None), -1), (dict(ptr=FAKE + 2), -1)])
def test_relation(b, over, code):  # noqa: F811
    rel = b._Packed(**{**PACKED, **over})
    assert fwd(b, rel) == code and b.load().tiga_last_error()
    assert bwd(b, over=over) == code
    assert b.load().tiga_mp_attention_packed_fwd_workspace(C.byref(rel)) == 0
    assert b.load().tiga_mp_attention_packed_bwd_workspace(C.byref(rel)) == 0


def test_arguments(b):  # noqa: F811
    E, W = b.TIGA_EINVAL, b.TIGA_EWORKSPACE
    bads = lambda: (None, view(b, data=None), view(b, data=FAKE + 8), view(b, row=60), view(b, head=-64))
    for name in ("q", "k", "v", "y"):
        for bad in bads():
            assert fwd(b, **{name: bad}) == E, (name, bad)
            assert bwd(b, **{name: bad}) == E, (name, bad)
    for name in ("dy", "dq", "dk", "dv"):
        for bad in bads()[1:]:
            assert bwd(b, **{name: bad}) == E, (name, bad)
    for bad in (view(b, row=0), view(b, head=0)):
        assert fwd(b, y=bad) == E and b"overlap" in b.load().tiga_last_error()
        for name in ("dq", "dk", "dv"):
            assert bwd(b, **{name: bad}) == E
    for name in ("k", "v"):
        assert fwd(b, **{name: view(b, row=1 << 23)}) == b.TIGA_EUNSUPPORTED
        assert bwd(b, **{name: view(b, row=1 << 23)}) == b.TIGA_EUNSUPPORTED
    for s in (0.0, -1.0, float("inf"), float("nan")):
        assert fwd(b, scale=s) == E and bwd(b, scale=s) == E
    assert fwd(b, lse=C.c_void_p(FAKE + 2)) == E and bwd(b, lse=FAKE + 2) == E and bwd(b, lse=0) == E
    for call in (fwd, bwd):
        assert call(b, ws=0) == E and call(b, ws=FAKE + 16) == E and call(b, n=0) == W
    # nothing to compute: no tensors needed
    for over in (dict(num_rows=0), dict(heads=0, kv_heads=0)):
        assert fwd(b, q=None, k=None, v=None, y=None, ws=0, n=0, **over) == 0
        assert bwd(b, over=over, q=None, k=None, v=None, y=None, dy=None, dq=None, dk=None, dv=None, lse=0, ws=0, n=0) == 0
    for which in ("fwd", "bwd"):  # source heads that nothing reads
        for over in (dict(heads=0), dict(heads=0, kv_heads=0), dict(num_rows=0), dict(batch=0), dict(batch=0, ptr=None)):
            assert getattr(b.load(), f"tiga_mp_attention_packed_{which}_workspace")(C.byref(b._Packed(**{**PACKED, **over}))) > 0
    # more tiles than one grid of threads counts
    many = dict(num_rows=(1 << 31) - 2048, heads=1, kv_heads=1, batch=(1 << 20) - 1)
    assert bwd(b, over=many) == b.TIGA_EUNSUPPORTED and b"tiles" in b.load().tiga_last_error()


@pytest.mark.parametrize("which", ["fwd", "bwd"])
def test_a_workspace_holds_every_smaller_call(b, which):  # noqa: F811
    size = lambda **o: getattr(b.load(), f"tiga_mp_attention_packed_{which}_workspace")(C.byref(b._Packed(**{**PACKED, **o})))
    for width in (64, 128):
        for big in (dict(num_rows=5000, batch=70, heads=32, kv_heads=8), dict(num_rows=40, batch=40, heads=8, kv_heads=8)):
            most = size(width=width, **big)
            for n in (1, 16, 17, 40, 129, 1000, 4999):
                for nb in (1, 2, 39, 70):
                    for h, hk in ((32, 8), (32, 4), (32, 1), (8, 8), (8, 2), (1, 1)):
                        if n <= big["num_rows"] and nb <= big["batch"] and h <= big["heads"] and hk <= big["kv_heads"]:
                            assert size(width=width, num_rows=n, batch=nb, heads=h, kv_heads=hk) <= most, (n, nb, h, hk)


def test_binding_refusals(b):  # noqa: F811
    q = torch.zeros(4, 10, 64, dtype=torch.float16)
    ptr = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(TypeError):
        b.tiga_mp_attention_packed_fwd(q, q, q, ptr)          # on the host
    with pytest.raises(ValueError):
        b.tiga_mp_attention_packed_fwd(q, q, q, ptr, layout="bhnd")
