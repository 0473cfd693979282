"""Paged attention calls whose launches would be too large are refused before any of them is made."""
import ctypes

import pytest

from paper_2511_09844_amd import binding as B

AT = 1 << 20  # an aligned address that no call here gets to read


def sizes(dtype, seqs, heads, hkv, hd, each, max_len):
    kv = B.PagedKv(AT, AT, hkv * 16 * hd, dtype, 16, 8, hkv, hd, 1 << 20, AT)
    rows = B.PagedRows(seqs, each, seqs * each, None, AT)
    return ctypes.byref(kv), ctypes.byref(rows), heads, max_len


def workspace(kv, rows, heads, max_len):
    return B.load().sd2_paged_attn_workspace_bytes(kv, rows, heads, max_len)


# the join of few rows (its kernel before it would fit), few rows by themselves, prompts, the join of prompts
LARGE = [(0, 4096, 1024, 256, 128, 48, 4000), (0, 4096, 1024, 1024, 128, 192, 64), (1, 4096, 1024, 1024, 64, 600, 64),
         (0, 4096, 1024, 1024, 128, 1000, 64), (1, 4096, 1024, 1024, 32, 64, 4000)]


@pytest.mark.parametrize("case", LARGE, ids=str)
def test_launches_too_large_are_refused(case):
    kv, rows, heads, max_len = sizes(*case)
    assert workspace(kv, rows, heads, max_len) == 0
    width = heads * case[4]
    assert B.load().sd2_paged_attn(kv, rows, AT, width, 2 * AT, width, heads, 0.1, max_len, AT, 1 << 62, None) == -1


@pytest.mark.parametrize("case", [(0, 1024, 1024, 256, 128, 48, 4000), (1, 4096, 64, 8, 64, 600, 4000),
                                  (1, 4096, 1024, 256, 64, 1, 4000)], ids=str)
def test_large_launches_are_not(case):
    assert workspace(*sizes(*case)) >= 256
