"""Paged attention on values at the edge of the definition, and how exact its sums are."""
import math

import pytest
import torch

from paged_ref import attend64, attend_bound, make_cache, rows_of

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
DTYPES = pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])


def queries(n, heads, hd, dtype, seed=1):
    return torch.randn(n, heads, hd, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def set_rows(pool, cache, b, positions, value):
    """Column 0 of these positions of sequence b."""
    table = cache.table[b].tolist()
    for j in positions:
        pool[table[j // cache.page_size], 0, :, j % cache.page_size, 0] = value


@DTYPES
@pytest.mark.parametrize("hkv,heads,hd", [(1, 2, 32), (2, 4, 64), (2, 2, 128)])
@pytest.mark.parametrize("rows", [1, 9, 40, 300])
@pytest.mark.parametrize("before", [0, 2500], ids=["short", "split"])
def test_scores_of_minus_infinity(dtype, hkv, heads, hd, rows, before):
    """Four sequences.  All scores -inf: the softmax of that is NaN, as in the definition, not the zeros of a row that
    reads nothing.  All but one, or all but the later half: those alone count.  No page: zeros."""
    n = before + rows
    cache = make_cache([n] * 4, dtype, hkv, hd, 16)
    ln, _ = rows_of([n] * 4, [rows] * 4, False)
    q = queries(4 * rows, heads, hd, dtype)
    q[..., 0] = q[..., 0].abs() + 0.5
    set_rows(cache.k, cache, 0, range(n), -math.inf)
    set_rows(cache.k, cache, 1, range(1, n), -math.inf)
    set_rows(cache.k, cache, 2, range((n + 1) // 2), -math.inf)
    cache.table[3] = -1
    got = cache.attend(q, ln, max_len=n).double().view(4, rows, heads, hd)
    ref, absv, spread = attend64(cache, q, [n] * 4, [rows] * 4)
    ref, absv = ref.view(4, rows, heads, hd), absv.view(4, rows, heads, hd)
    assert torch.isnan(got[0]).all()
    first = cache.v[int(cache.table[1, 0]), 0, :, 0].double().repeat_interleave(heads // hkv, 0)
    assert (got[1] == first).all()
    assert (got[3] == 0).all()
    reads = before + torch.arange(rows, device="cuda") >= (n + 1) // 2
    assert torch.isnan(got[2][~reads]).all()
    # (the sums of magnitudes that the bound goes by, without the infinite ones)
    plain = make_cache([n] * 4, dtype, hkv, hd, 16)
    spread = attend64(plain, q, [n] * 4, [rows] * 4)[2]
    assert ((got[2] - ref[2]).abs() <= attend_bound(ref[2], absv[2], spread, dtype, n, hd))[reads].all()


@DTYPES
@pytest.mark.parametrize("rows", [1, 33, 300])
@pytest.mark.parametrize("max_len", [None, 64], ids=["split", "whole"])
def test_minus_infinity_behind_missing_pages(dtype, rows, max_len):
    """The first page that is there begins at position 1600, which half of the rows reach, and its keys score -inf: zeros for
    the rows before it, which read nothing, and NaN for the others."""
    hkv, heads, hd, n = 2, 4, 64, 1600 + (rows + 1) // 2
    cache = make_cache([n, n], dtype, hkv, hd, 16)
    set_rows(cache.k, cache, 0, range(n), -math.inf)
    cache.table[0, :100] = -1
    cache.table[0, 7] = cache.n_pages  # (no page either)
    ln, _ = rows_of([n, n], [rows] * 2, False)
    q = queries(2 * rows, heads, hd, dtype)
    q[..., 0] = q[..., 0].abs() + 0.5
    got = cache.attend(q, ln, max_len=max_len)[:rows]
    reads = n - rows + torch.arange(rows, device="cuda") >= 1600
    assert torch.isnan(got[reads]).all() and (got[~reads] == 0).all() and reads.any()


@DTYPES
@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("rows", [3, 100])
def test_scale_zero_and_queries_that_are_no_numbers(dtype, hd, rows):
    """0 times an infinity or NaN is NaN; every other row is a mean."""
    n = rows + 70
    cache = make_cache([n], dtype, 2, hd, 16)
    q = queries(rows, 4, hd, dtype)
    q[0, 1, 3], q[2, 0, hd - 1], q[2, 3, 0] = math.nan, math.inf, -math.inf
    ln, _ = rows_of([n], [rows], False)
    got = cache.attend(q, ln, scale=0.0)
    odd = torch.zeros(rows, 4, dtype=torch.bool, device="cuda")
    odd[0, 1] = odd[2, 0] = odd[2, 3] = True
    assert torch.isnan(got[odd]).all()
    q[odd] = 0
    ref, absv, spread = attend64(cache, q, [n], [rows], scale=0.0)
    assert ((got.double() - ref).abs() <= attend_bound(ref, absv, spread, dtype, n, hd))[~odd].all()


@pytest.mark.parametrize("hkv,heads,hd", [(2, 4, 32), (2, 6, 64), (1, 8, 128), (2, 32, 64)])
@pytest.mark.parametrize("rows", [1, 2, 4])
@pytest.mark.parametrize("odd", [False, True], ids=["plain", "odd"])
def test_weights_of_few_bf16_rows(hkv, heads, hd, rows, odd):
    """The softmax's weights enter their product with v as two bf16 numbers each: the second, up to 2^-7 of the weight, is
    off by half a step of 2^-8, so the weight by 2^-15, and what a row is off by is its fp32 sums and its own
    rounding.  odd: with a NaN that only the last row reads, which such blocks are computed another way for."""
    lens = [20, 33, 64, 90, 300]
    cache = make_cache(lens, BF16, hkv, hd, 16)
    q = queries(rows * len(lens), heads, hd, BF16)
    ref, absv, spread = attend64(cache, q, lens, [rows] * len(lens))
    sums = attend_bound(ref, absv, spread, F32, max(lens), hd) + 2.0 ** -15 * absv
    bound = sums + 2.0 ** -8 * (ref.abs() + sums)
    if odd:
        for b, n in enumerate(lens):
            cache.v[int(cache.table[b, (n - 1) // 16]), 0, :, (n - 1) % 16, 0] = math.nan
    ln, _ = rows_of(lens, [rows] * len(lens), False)
    for max_len in (None, 64):  # split, and not
        err = (cache.attend(q, ln, max_len=max_len).double() - ref).abs()
        ok = err <= bound
        if odd:
            ok = ok.view(len(lens), rows, heads, hd)
            ok[:, -1, :, 0] = True
        assert ok.all(), float((err / bound).nan_to_num().max())


@DTYPES
@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("rows", [1, 6, 40, 200])
def test_infinite_values_stay_infinite(dtype, hd, rows):
    """Infinities of v that every row reads, beside weights of all sizes, 1 among them (a row that reads one key)."""
    lens = [rows + 150, rows]
    cache = make_cache(lens, dtype, 1, hd, 16)
    table = cache.table.tolist()
    for b, at in ((0, 7), (0, 100), (1, 0)):
        cache.v[table[b][at // 16], 0, :, at % 16, 1] = math.inf
        cache.v[table[b][at // 16], 0, :, at % 16, 2] = -math.inf
    cache.v[table[0][0], 0, :, 3, 2] = math.inf  # both signs
    ln, _ = rows_of(lens, [rows] * 2, False)
    q = queries(2 * rows, 3, hd, dtype)
    got = cache.attend(q, ln)
    assert (got[..., 1] == math.inf).all()
    assert torch.isnan(got[:rows, :, 2]).all() and (got[rows:, :, 2] == -math.inf).all()
    other = [c for c in range(hd) if c not in (1, 2)]
    ref, absv, spread = attend64(cache, q, lens, [rows] * 2)
    bound = attend_bound(ref, absv, spread, dtype, max(lens), hd)
    assert ((got.double() - ref).abs() <= bound)[..., other].all()
