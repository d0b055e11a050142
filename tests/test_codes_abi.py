"""Host side of the operators on 4-bit codes (no GPU): refusals before any launch, the cache structure's layout, sizes."""
import ctypes as C
import os
import re
import subprocess

import pytest

from conftest import ROOT


def test_cache_structure_matches_the_header(tmp_path):
    from paper_2608_18147_gb300 import native
    with open(os.path.join(ROOT, "include", "ecasq.h")) as f:
        body = re.search(r"typedef struct ecasq_cache \{([^}]*)\} ecasq_cache_t;", f.read()).group(1)
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    names = [n.strip(" *") for decl in body.split(";") if decl.strip() for n in decl.strip().split(None, 1)[1].split(",")]
    assert names == [n for n, _ in native.Cache._fields_]
    src = ["#include <stdio.h>", "#include <stddef.h>", '#include "ecasq.h"', "int main(void) {",
           'printf("%zu\\n", sizeof(ecasq_cache_t));']
    src += ['printf("%%zu\\n", offsetof(ecasq_cache_t, %s));' % n for n in names] + ["return 0;", "}"]
    c = tmp_path / "layout.c"
    c.write_text("\n".join(src))
    subprocess.run(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), str(c), "-o", str(tmp_path / "layout")], check=True)
    got = [int(v) for v in subprocess.run([str(tmp_path / "layout")], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [C.sizeof(native.Cache)] + [getattr(native.Cache, n).offset for n in names]


V = 1 << 20  # stands for a device address: nothing is launched with it


def test_matvec_and_pack_refusals():
    from paper_2608_18147_gb300 import native
    L = native.lib()
    good = dict(x=V, x_row=300, type=native.BF16, b=2, codes=V, code_row=192, levels=V, m=16, scales=V, scale_row=10,
                scale_type=native.F32, n=5, k=300, group=32, y=V, y_row=5, status=None, stream=None)
    assert L.ecasq_matvec(*dict(good, b=0).values()) == native.OK
    for change in (dict(x=None), dict(type=3), dict(type=-1), dict(b=-1), dict(codes=None), dict(codes=V + 8), dict(code_row=191),
                   dict(code_row=128), dict(code_row=200), dict(levels=None), dict(m=0), dict(m=17), dict(scales=None),
                   dict(scale_row=9), dict(scale_type=native.F16), dict(scale_type=7), dict(n=0), dict(n=1 << 31), dict(k=0),
                   dict(k=1 << 31), dict(group=0), dict(group=16), dict(group=40), dict(group=-32), dict(y=None), dict(x_row=299),
                   dict(y_row=4)):
        assert L.ecasq_matvec(*dict(good, **change).values()) == native.EINVAL, change
    good = dict(idx=V, idx_row=300, n=4, k=300, codes=V, code_row=192, stream=None)
    for change in (dict(idx=None), dict(idx_row=299), dict(n=0), dict(k=0), dict(codes=None), dict(codes=V + 4), dict(code_row=191),
                   dict(code_row=200), dict(code_row=128)):
        assert L.ecasq_pack(*dict(good, **change).values()) == native.EINVAL, change


def plain(native, **change):
    f = dict(rows=V, levels=None, row_page=16 * 128, row_slot=128, row_head=64, level_page=0, level_slot=0, level_head=0, pages=9,
             page_size=16, heads=2, d=64, type=native.BF16, levels_n=0, reserved=0)
    return native.Cache(*dict(f, **change).values())


def coded(native, **change):
    f = dict(rows=V, levels=V, row_page=16 * 64, row_slot=64, row_head=32, level_page=256, level_slot=16, level_head=8, pages=9,
             page_size=16, heads=2, d=64, type=native.BF16, levels_n=8, reserved=0)
    return native.Cache(*dict(f, **change).values())


BAD_CACHES = [dict(rows=None), dict(rows=V + 8), dict(row_page=2050), dict(row_slot=129), dict(row_head=60), dict(pages=0),
              dict(pages=1 << 62), dict(page_size=0), dict(heads=0), dict(d=0), dict(d=60), dict(d=264), dict(type=3), dict(levels_n=4)]
BAD_CODED = [dict(levels=None), dict(levels=V + 8), dict(level_page=12), dict(level_slot=9), dict(level_head=1), dict(d=48),
             dict(type=0), dict(levels_n=9), dict(row_slot=72)]


def test_cache_write_refusals():
    from paper_2608_18147_gb300 import native
    L = native.lib()
    good = dict(x=V, x_type=native.F32, n=3, x_row=128, x_head=64, Q=V, s=8, m=V, slots=V, cache=None, seed=1, status=None,
                stream=None)

    def call(cache, **change):
        return L.ecasq_cache_write(*dict(good, cache=C.byref(cache), **change).values())

    assert call(coded(native), n=0) == native.OK
    for change in (dict(x=None), dict(x_type=native.F16), dict(x_type=5), dict(n=-1), dict(Q=None), dict(s=0), dict(s=9), dict(slots=None)):
        assert call(coded(native), **change) == native.EINVAL, change
    assert call(plain(native)) == native.EINVAL
    assert L.ecasq_cache_write(*good.values()) == native.EINVAL
    for change in BAD_CACHES + BAD_CODED:
        assert call(coded(native, **change)) == native.EINVAL, change


def test_attend_refusals():
    from paper_2608_18147_gb300 import native
    L = native.lib()
    need = L.ecasq_workspace_size_attend(2, 4, 2, 64, 160)
    good = dict(q=V, q_row=256, q_head=64, b=2, heads=4, k=None, v=None, table=V, table_row=10, lengths=V, starts=None,
                max_len=160, scale=0.1, out=V, out_row=256, out_head=64, lse=None, ws=V, ws_bytes=need, status=None, stream=None)

    def call(k, v, **change):
        return L.ecasq_attend(*dict(good, k=C.byref(k), v=C.byref(v), **change).values())

    assert call(plain(native), plain(native), b=0) == native.OK
    for change in (dict(q=None), dict(b=-1), dict(heads=0), dict(heads=3), dict(table=None), dict(table_row=9), dict(lengths=None),
                   dict(max_len=-1), dict(max_len=161), dict(max_len=1 << 31), dict(out=None)):
        assert call(plain(native), plain(native), **change) == native.EINVAL, change
    for change in BAD_CACHES:
        assert call(plain(native, **change), plain(native)) == native.EINVAL, change
        assert call(plain(native), plain(native, **change)) == native.EINVAL, change
    for change in BAD_CACHES + BAD_CODED:
        assert call(coded(native), coded(native, **change)) == native.EINVAL, change
    for change in (dict(pages=8), dict(page_size=8), dict(heads=4), dict(d=56), dict(type=native.F16)):
        assert call(plain(native), plain(native, **change)) == native.EINVAL, change
    assert call(plain(native), coded(native)) == native.EINVAL
    assert call(coded(native), coded(native, levels_n=16)) == native.EINVAL
    assert L.ecasq_attend(*good.values()) == native.EINVAL


def test_attend_workspace():
    """A short cache needs none; more keys, sequences or heads never need less; bad sizes need none."""
    from paper_2608_18147_gb300 import native
    size = native.lib().ecasq_workspace_size_attend
    assert size(1, 8, 8, 128, 1) == 0
    assert size(1, 8, 8, 128, 0) == 0
    for bad in ((-1, 8, 8, 128, 100), (1, 0, 8, 128, 100), (1, 8, 3, 128, 100), (1, 8, 8, 0, 100), (1, 8, 8, 128, -1)):
        assert size(*bad) == 0
    assert size(1, 8, 8, 128, 100000) < 64 << 20


def test_binding_refuses_tensors_of_the_host():
    torch = pytest.importorskip("torch")
    from paper_2608_18147_gb300 import native
    z = torch.zeros(4, 64, dtype=torch.uint8)
    f = torch.zeros(4, 64)
    rows = torch.zeros(2, 16, 2, 64)
    i = torch.zeros(4, 1, dtype=torch.int32)
    for fn, args in ((native.ecasq_pack, (z,)), (native.ecasq_matvec, (f, z, f[0, :16], f, 32)),
                     (native.ecasq_cache_write, (rows, f, None, i, rows, rows, 1)),
                     (native.ecasq_attend, (rows[0], rows, rows, i, i))):
        with pytest.raises(native.EcasqError) as err:
            fn(*args)
        assert err.value.code == native.EINVAL
