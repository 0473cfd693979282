"""Refusals of the entry points for caches of 8 bits and for windows, before anything reaches a GPU, and the structures'
layouts."""
import ctypes
import os
import subprocess

import pytest

from paper_2511_09844_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
AT = 1 << 20  # an aligned address that no call here gets to read


def scaled(**kw):
    c = dict(k=AT, v=AT, page_stride=4 * 16 * 64, dtype=1, page_size=16, n_pages=8, n_kv_heads=4, head_dim=64, max_pages=4,
             table=AT, scales=AT, scale_stride=8)
    c.update(kw)
    return B.PagedScaled(B.PagedKv(*(c[f[0]] for f in B.PagedKv._fields_)), c["scales"], c["scale_stride"])


def rows(**kw):
    c = dict(nseq=2, max_rows=1, total_rows=2, row_off=None, lens=AT)
    c.update(kw)
    return B.PagedRows(*(c[f[0]] for f in B.PagedRows._fields_))


def pages(**kw):
    c = dict(page_size=16, n_pages=8, max_seqs=4, max_pages=4, table=AT, refs=AT, n_arrays=1, blocks=2, row_bytes=-64, data=AT)
    c.update(kw)
    p = B.Pages(c["page_size"], c["n_pages"], c["max_seqs"], c["max_pages"], c["table"], c["refs"], c["n_arrays"])
    p.arrays[0] = B.PageArray(c["data"], c["blocks"], c["row_bytes"])
    return p


def attn(lib, c, r, fn="sd2_paged_attn_scaled", q=AT, qs=512, out=2 * AT, os_=512, heads=8, scale=0.125, max_len=64, window=0,
         sinks=0, ws=AT, n=1 << 30):
    return getattr(lib, fn)(ctypes.byref(c), ctypes.byref(r), q, qs, out, os_, heads, scale, max_len, window, sinks, ws, n, None)


BAD = [dict(k=None), dict(v=AT + 8), dict(page_stride=4 * 16 * 64 - 16), dict(page_stride=4 * 16 * 64 + 8), dict(dtype=2),
       dict(page_size=8), dict(n_pages=0), dict(n_kv_heads=0), dict(head_dim=96), dict(max_pages=0), dict(table=None),
       dict(scales=None), dict(scales=AT + 1), dict(scale_stride=6), dict(scale_stride=9), dict(scale_stride=-8),
       dict(scale_stride=(1 << 40) + 2)]


@pytest.mark.parametrize("kw", BAD, ids=str)
def test_cache_refused(kw):
    lib, c, r = B.load(), scaled(**kw), rows()
    assert attn(lib, c, r) == -1
    assert lib.sd2_paged_attn_scaled_workspace_bytes(ctypes.byref(c), ctypes.byref(r), 8, 64, 0, 0) == 0
    assert lib.sd2_paged_append_scaled(ctypes.byref(c), ctypes.byref(r), AT, 256, AT, 256, None) == -1


@pytest.mark.parametrize("kw", [dict(nseq=-1), dict(max_rows=0, total_rows=0), dict(total_rows=3), dict(lens=None), dict(row_off=AT + 1)], ids=str)
def test_rows_refused(kw):
    lib, c, r = B.load(), scaled(), rows(**kw)
    assert attn(lib, c, r) == -1 and attn(lib, c.kv, r, "sd2_paged_attn_window") == -1
    assert lib.sd2_paged_attn_scaled_workspace_bytes(ctypes.byref(c), ctypes.byref(r), 8, 64, 0, 0) == 0
    assert lib.sd2_paged_append_scaled(ctypes.byref(c), ctypes.byref(r), AT, 256, AT, 256, None) == -1


@pytest.mark.parametrize("fn", ["sd2_paged_attn_scaled", "sd2_paged_attn_window"])
def test_arguments_refused(fn):
    lib, r = B.load(), rows()
    c = scaled() if fn.endswith("scaled") else scaled().kv
    size = getattr(lib, fn + "_workspace_bytes")
    for kw in [dict(q=None), dict(q=AT + 8), dict(qs=504), dict(qs=516), dict(out=None), dict(out=AT), dict(os_=8), dict(heads=0),
               dict(heads=6), dict(heads=1028), dict(scale=float("nan")), dict(max_len=0), dict(max_len=65), dict(ws=None),
               dict(ws=AT + 64), dict(n=0), dict(window=-1), dict(window=(1 << 30) + 1), dict(window=1, sinks=-1),
               dict(window=1, sinks=(1 << 30) + 1)]:
        assert attn(lib, c, r, fn, **kw) == -1, kw
    for args in [(8, 64, -1, 0), (8, 64, (1 << 30) + 1, 0), (8, 64, 1, -1), (8, 64, 1, (1 << 30) + 1), (6, 64, 1, 0), (8, 65, 1, 0)]:
        assert size(ctypes.byref(c), ctypes.byref(r), *args) == 0, args
    assert size(ctypes.byref(c), ctypes.byref(r), 8, 64, 1 << 30, 1 << 30) > 0
    none = rows(nseq=0, total_rows=0, lens=None)
    assert attn(lib, c, none, fn, q=None, out=None) == 0
    if fn.endswith("scaled"):
        for args in [(None, 256, AT, 256), (AT, 248, AT, 256), (AT, 256, AT + 4, 256), (AT, 256, AT, 260)]:
            assert lib.sd2_paged_append_scaled(ctypes.byref(c), ctypes.byref(r), *args, None) == -1, args
        assert lib.sd2_paged_append_scaled(ctypes.byref(c), ctypes.byref(none), None, 0, None, 0, None) == 0
        wide = scaled(dtype=0)  # fp32 rows: 16-byte units of four
        assert attn(lib, wide, r, qs=514) == -1
    many = rows(total_rows=(1 << 29) + 1, max_rows=1 << 30, row_off=AT)
    assert attn(lib, c, many, fn) == -1 and size(ctypes.byref(c), ctypes.byref(many), 8, 64, 4, 0) == 0


@pytest.mark.parametrize("kw", [dict(row_bytes=-1), dict(row_bytes=-3), dict(row_bytes=-(1 << 20) - 2), dict(row_bytes=0),
                                dict(row_bytes=-2 ** 31), dict(blocks=0), dict(data=AT + 8)], ids=str)
def test_records_refused(kw):
    lib, p = B.load(), pages(**kw)
    assert lib.sd2_pages_workspace_bytes(ctypes.byref(p)) == 0
    assert lib.sd2_pages_slide(ctypes.byref(p), 1, AT, 1, 0, None) == -1


def test_slide_refused():
    lib, p = B.load(), pages()
    assert lib.sd2_pages_workspace_bytes(ctypes.byref(p)) > 0
    for args in [(-1, AT, 1, 0), (5, AT, 1, 0), (1, None, 1, 0), (1, AT + 2, 1, 0), (1, AT, 0, 0), (1, AT, -1, 0), (1, AT, 1, -1),
                 (1, AT, (1 << 30) + 1, 0), (1, AT, 1, (1 << 30) + 1)]:
        assert lib.sd2_pages_slide(ctypes.byref(p), *args, None) == -1, args
    assert lib.sd2_pages_slide(None, 1, AT, 1, 0, None) == -1
    assert lib.sd2_pages_slide(ctypes.byref(p), 0, None, 1, 0, None) == 0


def test_struct_layout_matches_the_header(tmp_path):
    prog, exe = tmp_path / "layout.c", tmp_path / "layout"
    prog.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "sd2.h"\nint main(void) { printf("%zu", sizeof(sd2_paged_scaled));'
                    + "".join(f'printf(" %zu", offsetof(sd2_paged_scaled, {f[0]}));' for f in B.PagedScaled._fields_) + "return 0; }\n")
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(prog), "-o", str(exe)])
    got = list(map(int, subprocess.check_output([str(exe)]).decode().split()))
    assert got == [ctypes.sizeof(B.PagedScaled)] + [getattr(B.PagedScaled, f[0]).offset for f in B.PagedScaled._fields_]
