"""sd2_paged_attn refuses a q and an out that share an element, before anything reaches a GPU.  (Pairs that share none
are not called here: their addresses are made up.)"""
import ctypes

import pytest

from paper_2511_09844_amd import binding as B

AT = 1 << 30


def shared(d, qs, os_, width, rows):
    """By the elements themselves: q's first at 0, out's at d."""
    q = {r * qs + i for r in range(rows) for i in range(width)}
    return any(d + r * os_ + i in q for r in range(rows) for i in range(width))


@pytest.mark.parametrize("dtype", [0, 1], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows", [1, 2, 3])
@pytest.mark.parametrize("qs,os_", [(64, 64), (160, 160), (160, 96), (96, 160)])
def test_operands_that_share_elements_are_refused(dtype, rows, qs, os_):
    lib, width, size = B.load(), 64, 2 if dtype else 4
    kv = B.PagedKv(1 << 20, 1 << 20, 2 * 16 * 32, dtype, 16, 8, 2, 32, 4, 1 << 20)
    r = B.PagedRows(rows, 1, rows, None, 1 << 20)
    seen = 0
    for d in range(-4 * 160, 4 * 160 + 1, 8):
        if shared(d, qs, os_, width, rows):
            seen += 1
            args = AT, qs, AT + d * size, os_, 2, 0.1, 64, 1 << 20, 1 << 20, None
            assert lib.sd2_paged_attn(ctypes.byref(kv), ctypes.byref(r), *args) == -1, d
    assert seen >= 15


def test_operands_far_apart_in_rows_are_refused_too():
    """Extents past 64 bits."""
    lib, far = B.load(), 1 << 40
    kv = B.PagedKv(1 << 20, 1 << 20, 2 * 16 * 32, 0, 16, 8, 2, 32, 4, 1 << 20)
    r = B.PagedRows(4096, 1 << 18, 1 << 30, None, 1 << 20)
    for q, out in ((AT, AT + 128), (AT + 128, AT), (AT, AT)):
        assert lib.sd2_paged_attn(ctypes.byref(kv), ctypes.byref(r), q, far, out, far, 2, 0.1, 64, 1 << 20, 1 << 40, None) == -1
