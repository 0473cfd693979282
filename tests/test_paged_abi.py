"""Refusals of the paged entry points, before anything reaches a GPU, and the structures' layouts."""
import ctypes
import os
import subprocess

import pytest

from paper_2511_09844_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
AT = 1 << 20  # an aligned address that no call here gets to read


def pages(**kw):
    c = dict(page_size=16, n_pages=8, max_seqs=4, max_pages=4, table=AT, refs=AT, n_arrays=1, blocks=2, row_bytes=64, data=AT)
    c.update(kw)
    p = B.Pages(c["page_size"], c["n_pages"], c["max_seqs"], c["max_pages"], c["table"], c["refs"], c["n_arrays"])
    p.arrays[0] = B.PageArray(c["data"], c["blocks"], c["row_bytes"])
    return p


def kv(**kw):
    c = dict(k=AT, v=AT, page_stride=4 * 16 * 64, dtype=1, page_size=16, n_pages=8, n_kv_heads=4, head_dim=64, max_pages=4,
             table=AT)
    c.update(kw)
    return B.PagedKv(*(c[f[0]] for f in B.PagedKv._fields_))


def rows(**kw):
    c = dict(nseq=2, max_rows=1, total_rows=2, row_off=None, lens=AT)
    c.update(kw)
    return B.PagedRows(*(c[f[0]] for f in B.PagedRows._fields_))


BAD_PAGES = [dict(page_size=8), dict(page_size=24), dict(page_size=2048), dict(n_pages=0), dict(n_pages=(1 << 24) + 1),
             dict(max_seqs=0), dict(max_seqs=4097), dict(max_pages=0), dict(max_pages=1 << 27), dict(table=None),
             dict(refs=None), dict(refs=AT + 2), dict(n_arrays=0), dict(n_arrays=9), dict(data=None), dict(data=AT + 8),
             dict(blocks=0), dict(blocks=65537), dict(row_bytes=8), dict(row_bytes=24), dict(row_bytes=65552)]


@pytest.mark.parametrize("kw", BAD_PAGES, ids=str)
def test_pages_refused(kw):
    lib, p, n = B.load(), pages(**kw), (ctypes.c_int32 * 1)(0)
    assert lib.sd2_pages_workspace_bytes(ctypes.byref(p)) == 0
    assert lib.sd2_pages_reserve(ctypes.byref(p), 1, AT, AT, None, None, AT, 1 << 30, None) == -1
    assert lib.sd2_pages_fork(ctypes.byref(p), 1, n, n, None) == -1
    assert lib.sd2_pages_trim(ctypes.byref(p), 1, AT, None) == -1
    assert lib.sd2_pages_compact(ctypes.byref(p), None, AT, 1 << 30, None) == -1


def test_page_calls_refused():
    lib, p = B.load(), pages()
    need = lib.sd2_pages_workspace_bytes(ctypes.byref(p))
    assert need > 0
    ref = ctypes.byref(p)
    for args in [(-1, AT, AT, None, None, AT, need), (5, AT, AT, None, None, AT, need), (1, None, AT, None, None, AT, need),
                 (1, AT, None, None, None, AT, need), (1, AT, AT, None, None, None, need),
                 (1, AT, AT, None, None, AT + 16, need), (1, AT, AT, None, None, AT, need - 1)]:
        assert lib.sd2_pages_reserve(ref, *args, None) == -1, args
    assert lib.sd2_pages_reserve(ref, 0, None, None, None, None, AT, need, None) == 0
    assert lib.sd2_pages_trim(ref, 5, AT, None) == -1 and lib.sd2_pages_trim(ref, 1, None, None) == -1
    assert lib.sd2_pages_trim(ref, 0, None, None) == 0
    assert lib.sd2_pages_compact(ref, None, AT, need - 1, None) == -1
    for fn in (lib.sd2_pages_reserve, lib.sd2_pages_compact):
        args = (1, AT, AT, None, None) if fn is lib.sd2_pages_reserve else (None,)
        assert fn(None, *args, AT, need, None) == -1


@pytest.mark.parametrize("src,dst", [([0], [0]), ([0, 0], [1, 1]), ([0, 1], [1, 2]), ([4], [1]), ([0], [4]), ([-1], [1]),
                                     ([0], [-1]), ([0] * 5, [1, 2, 3, 0, 0])])
def test_forks_refused(src, dst):
    lib, p = B.load(), pages()
    arr = ctypes.c_int32 * len(src)
    assert lib.sd2_pages_fork(ctypes.byref(p), len(src), arr(*src), arr(*dst), None) == -1
    assert lib.sd2_pages_fork(ctypes.byref(p), 0, None, None, None) == 0
    assert lib.sd2_pages_fork(ctypes.byref(p), 1, None, arr(*dst), None) == -1


def attn(lib, c, r, q=AT, qs=512, out=2 * AT, os_=512, heads=8, scale=0.125, max_len=64, ws=AT, n=1 << 30):
    return lib.sd2_paged_attn(ctypes.byref(c), ctypes.byref(r), q, qs, out, os_, heads, scale, max_len, ws, n, None)


BAD_KV = [dict(k=None), dict(v=None), dict(k=AT + 8), dict(page_stride=4 * 16 * 64 - 8), dict(page_stride=4 * 16 * 64 + 4),
          dict(dtype=2), dict(dtype=-1), dict(page_size=0), dict(page_size=48), dict(n_pages=0), dict(n_kv_heads=0),
          dict(n_kv_heads=1025), dict(head_dim=96), dict(head_dim=256), dict(max_pages=0), dict(max_pages=1 << 28),
          dict(table=None), dict(table=AT + 1)]


@pytest.mark.parametrize("kw", BAD_KV, ids=str)
def test_cache_refused(kw):
    lib, c, r = B.load(), kv(**kw), rows()
    assert attn(lib, c, r) == -1
    assert lib.sd2_paged_attn_workspace_bytes(ctypes.byref(c), ctypes.byref(r), 8, 64) == 0
    assert lib.sd2_paged_append(ctypes.byref(c), ctypes.byref(r), AT, 256, AT, 256, None) == -1


BAD_ROWS = [dict(nseq=-1), dict(nseq=4097, total_rows=4097), dict(max_rows=0, total_rows=0), dict(total_rows=-1),
            dict(total_rows=3), dict(lens=None), dict(lens=AT + 2), dict(row_off=AT + 1)]


@pytest.mark.parametrize("kw", BAD_ROWS, ids=str)
def test_rows_refused(kw):
    lib, c, r = B.load(), kv(), rows(**kw)
    assert attn(lib, c, r) == -1
    assert lib.sd2_paged_attn_workspace_bytes(ctypes.byref(c), ctypes.byref(r), 8, 64) == 0
    assert lib.sd2_paged_append(ctypes.byref(c), ctypes.byref(r), AT, 256, AT, 256, None) == -1


def test_attn_and_append_arguments_refused():
    lib, c, r = B.load(), kv(), rows()
    for kw in [dict(q=None), dict(q=AT + 8), dict(qs=504), dict(qs=516), dict(out=None), dict(os_=8), dict(heads=0),
               dict(heads=6), dict(heads=1028), dict(scale=float("nan")), dict(scale=float("inf")), dict(max_len=0),
               dict(max_len=65), dict(ws=None), dict(ws=AT + 64), dict(n=0)]:
        assert attn(lib, c, r, **kw) == -1, kw
    # more query vectors of one sequence and KV head than 2^30
    many = rows(total_rows=(1 << 29) + 1, max_rows=1 << 30, row_off=AT)
    assert attn(lib, c, many) == -1
    assert lib.sd2_paged_attn_workspace_bytes(ctypes.byref(c), ctypes.byref(many), 8, 64) == 0
    for args in [(None, 256, AT, 256), (AT, 248, AT, 256), (AT, 256, AT + 4, 256), (AT, 256, AT, 260)]:
        assert lib.sd2_paged_append(ctypes.byref(c), ctypes.byref(r), *args, None) == -1, args
    # nothing to do is no error
    none = rows(nseq=0, total_rows=0, lens=None)
    assert attn(lib, c, none, q=None, out=None) == 0
    assert lib.sd2_paged_append(ctypes.byref(c), ctypes.byref(none), None, 0, None, 0, None) == 0
    assert attn(lib, c, rows(total_rows=0, row_off=AT)) == 0
    for r in (none, rows(total_rows=0, row_off=AT), rows(nseq=0, total_rows=0, row_off=AT, max_rows=2 ** 31 - 1)):
        assert lib.sd2_paged_attn_workspace_bytes(ctypes.byref(c), ctypes.byref(r), 8, 64) > 0


def test_paged_struct_layouts_match_the_header(tmp_path):
    structs = {"sd2_page_array": B.PageArray, "sd2_pages": B.Pages, "sd2_paged_kv": B.PagedKv, "sd2_paged_rows": B.PagedRows}
    body = "".join(f'printf("%zu", sizeof({c}));' + "".join(f'printf(" %zu", offsetof({c}, {f[0]}));' for f in s._fields_)
                   + 'printf("\\n");' for c, s in structs.items())
    prog, exe = tmp_path / "layout.c", tmp_path / "layout"
    prog.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "sd2.h"\nint main(void) {' + body + "return 0; }\n")
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(prog), "-o", str(exe)])
    got = [list(map(int, line.split())) for line in subprocess.check_output([str(exe)]).decode().splitlines()]
    for line, s in zip(got, structs.values()):
        assert line == [ctypes.sizeof(s)] + [getattr(s, f[0]).offset for f in s._fields_], s


def test_paged_handles_refused():
    import sd2_inputs as si
    lib, cfg, h = B.load(), B.config_of(si.TINY), B.P()
    ref = ctypes.byref(cfg)

    def size(page, n, c=cfg):
        return lib.sd2_create_paged_bytes(ctypes.byref(c), ctypes.byref(B.Paging(page, n)))

    assert size(16, 8) > 0 and size(64, 8) > size(32, 8)
    # a page holds page_size rows of k and v in every layer and KV head of both models
    per = 16 * 2 * 4 * (4 * 8 * 32 + 2 * 4 * 32)
    assert 1000 * per <= size(16, 1008) - size(16, 8) <= 1000 * (per + 64)
    bad = [(0, 8), (8, 8), (48, 8), (2048, 8), (16, 0), (16, -1), (16, (1 << 24) + 1)]
    for page, n in bad:
        assert size(page, n) == 0
        pg = B.Paging(page, n)
        assert lib.sd2_create_paged(ref, None, None, None, ctypes.byref(pg), None, 0, None, ctypes.byref(h)) == -1
    assert lib.sd2_create_paged_bytes(ref, None) == 0
    mlp = B.config_of(si.TINY, steering=B.STEER_MLP)
    assert size(16, 8, mlp) == 0
    pg = B.Paging(16, 8)
    assert lib.sd2_create_paged(ctypes.byref(mlp), None, None, None, ctypes.byref(pg), None, 0, None, ctypes.byref(h)) == -1
    assert lib.sd2_create_paged(ref, None, None, None, ctypes.byref(pg), None, 0, None, None) == -1
    assert lib.sd2_fork(None, 0, 1) == -1 and lib.sd2_release(None, 0) == -1 and lib.sd2_compact(None, None) == -1
