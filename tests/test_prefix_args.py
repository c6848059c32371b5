"""Host-side checks of attention behind shared prefixes: every call returns before anything reaches a device."""
import ctypes as C
import os
import subprocess

import pytest

from tests.test_relattn_args import FAKE, ROOT, b, view  # noqa: F401


def cache(b, **over):
    base = dict(num_pages=64, page_size=16, kv_heads=2, width=64, dtype=0, batch=3, table_width=8, k=view(b), v=view(b),
                table=FAKE, length=FAKE)
    return b._Cache(**{**base, **over})


def call(b, c=None, groups=2, ptr=FAKE, len=FAKE, prefix=0, num_dst=3, dst_ptr=FAKE, heads=4, q=0, y=0, scale=0.125, lse=None,
         ws=FAKE, n=1 << 40):
    p = b._Prefix(groups, ptr, len)
    r = lambda x: C.byref(view(b)) if x == 0 else C.byref(x) if x is not None else None
    return b.load().tiga_mp_attention_prefix_fwd(C.byref(c or cache(b)), C.byref(p) if prefix == 0 else None, num_dst,
                                                 C.c_void_p(dst_ptr), heads, r(q), scale, r(y), lse, C.c_void_p(ws), n, None)


def test_struct_layout_matches_the_header(tmp_path, b):  # noqa: F811
    s = b._Prefix
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "tiga_mp.h"\nint main(void) {\n  printf("%zu", sizeof(tiga_prefix));\n'
                   + "".join(f'  printf(" %zu", offsetof(tiga_prefix, {f}));\n' for f, _ in s._fields_) + "  return 0;\n}\n")
    subprocess.check_call(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "l")])
    got = [int(x) for x in subprocess.check_output([str(tmp_path / "l")]).split()]
    assert got == [C.sizeof(s)] + [getattr(s, f).offset for f, _ in s._fields_]


def test_arguments(b):  # noqa: F811
    E, U, W = b.TIGA_EINVAL, b.TIGA_EUNSUPPORTED, b.TIGA_EWORKSPACE
    assert call(b, prefix=None) == E and call(b, groups=-1) == E and call(b, groups=1 << 16) == U
    assert call(b, ptr=None) == E and call(b, len=None) == E and call(b, ptr=FAKE + 1) == E and call(b, len=FAKE + 2) == E
    assert call(b, c=cache(b, page_size=12)) == E and call(b, c=cache(b, width=80)) == U
    assert call(b, heads=5) == E and call(b, num_dst=-1) == E and call(b, num_dst=1 << 31) == U
    assert call(b, dst_ptr=None) == E and call(b, c=cache(b, table=None)) == E and call(b, c=cache(b, num_pages=0)) == E
    for s in (0.0, float("nan"), float("inf")):
        assert call(b, scale=s) == E
    for bad in (None, view(b, data=FAKE + 8), view(b, row=12)):
        assert call(b, q=bad) == E and call(b, y=bad) == E
    assert call(b, y=view(b, row=0)) == E and call(b, y=view(b, row=128)) == E      # overlaps; in q's place with other strides
    assert call(b, lse=C.c_void_p(FAKE + 2)) == E
    assert call(b, ws=0) == E and call(b, ws=FAKE + 16) == E and call(b, n=0) == W
    # nothing to do: no arrays needed
    assert call(b, num_dst=0, q=None, y=None, ws=0, n=0) == 0 and call(b, c=cache(b, batch=0), q=None, y=None, ws=0, n=0) == 0


@pytest.mark.parametrize("width", [64, 128])
def test_a_workspace_holds_every_smaller_call(b, width):  # noqa: F811
    def size(num_dst, heads, groups, **over):
        p = b._Prefix(groups, FAKE, FAKE)
        return b.load().tiga_mp_attention_prefix_fwd_workspace(C.byref(cache(b, width=width, **over)), C.byref(p), num_dst, heads)

    most = size(300, 32, 9, kv_heads=8, batch=64, table_width=600)
    for n in (1, 7, 16, 17, 64, 299):
        for h, hk in ((32, 8), (32, 1), (8, 8), (4, 2)):
            for groups in (0, 1, 9):
                for batch, table in ((64, 600), (1, 600), (64, 3), (17, 1)):
                    assert size(n, h, groups, kv_heads=hk, batch=batch, table_width=table) <= most
    paged = b.load().tiga_mp_attention_paged_fwd_workspace(C.byref(cache(b, width=width)), 300, 4)
    assert size(300, 4, 0) >= paged and size(300, 4, 70000) == 0
