"""Paged caches of 8 bits on the GPU: appending, attention, pages that go along with their scales."""
import math

import pytest
import torch

from paged_ref import PageModel, rows_of
from paged_scaled_ref import append64, check, make_scaled, values64

pytestmark = pytest.mark.gpu
T = {"bf16": torch.bfloat16, "f32": torch.float32}


def rand(*shape, dtype, seed, by=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * by).to(dtype).cuda()


def same_pools(cache, pools, scales):
    """Every byte but the sign of zeros and NaN."""
    for got, want in zip((cache.k, cache.v), pools):
        got = got.double().cpu()
        assert torch.equal(got.isnan(), want.isnan())
        assert torch.equal(got.nan_to_num(0), want.nan_to_num(0))
    assert torch.equal(cache.scales.view(torch.uint8).cpu(), scales)


# lens and rows of each sequence: whole prompts, single rows at every place of a block, blocks' ends, rows before position 0
APPENDS = [([1], [1]), ([16, 17, 1, 33], [1, 1, 1, 1]), ([40, 7, 100, 16], [40, 7, 100, 16]), ([50, 31, 90], [3, 17, 61]),
           ([5, 0, 20, 64], [0, 0, 20, 1]), ([3, 40], [5, 2]), ([130, 200], [20, 190])]


@pytest.mark.parametrize("dtype", list(T))
@pytest.mark.parametrize("hd,hkv,page", [(32, 1, 16), (64, 3, 32), (128, 2, 64), (64, 8, 256)])
@pytest.mark.parametrize("lens,rows", APPENDS, ids=str)
def test_append(dtype, hd, hkv, page, lens, rows):
    cache = make_scaled(lens, hkv, hd, page, layers=2, seed=len(lens))
    n = sum(rows)
    # magnitudes from far below what the blocks hold to far above
    by = torch.exp2(torch.randint(-20, 20, (n, hkv, 1), generator=torch.Generator().manual_seed(5)).float()).cuda()
    k, v = (rand(n, hkv, hd, dtype=torch.float32, seed=s).mul(by).to(T[dtype]) for s in (1, 2))
    want = append64(cache, k, v, lens, rows, layer=1)
    dl, off = rows_of(lens, rows, packed=min(rows) < max(rows))
    cache.append(k, v, dl, layer=1, row_off=off)
    same_pools(cache, *want)
    cache.append(k, v, dl, layer=1, row_off=off)  # the same rows again: nothing grows
    same_pools(cache, *append64(cache, k, v, lens, rows, layer=1))


@pytest.mark.parametrize("dtype", list(T))
@pytest.mark.parametrize("lens", [[20], [16, 5]])
def test_append_of_what_has_no_number(dtype, lens):
    cache = make_scaled(lens, 2, 64, 16)
    k, v = (rand(sum(lens), 2, 64, dtype=T[dtype], seed=s) for s in (3, 4))
    top = torch.finfo(T[dtype]).max
    k[0, 0, :4] = torch.tensor([math.inf, -math.inf, math.nan, -0.0])
    k[1, 1], v[1, 0] = 0.0, math.inf                       # a row of zeros; one without a finite value
    k[2, 0, 5], v[2, 1, 6], v[3, 1] = top, -top, 1e-38   # beyond what a power reaches; below
    k[4, 0, 0], v[4, 0, 1] = 448.0, 464.0                # ties at the end of the range
    want = append64(cache, k, v, lens, lens)
    dl, off = rows_of(lens, lens, packed=len(lens) > 1)
    cache.append(k, v, dl, row_off=off)
    same_pools(cache, *want)


def test_append_row_by_row_holds_what_one_call_does():
    """Powers that grow row by row: numbers of 2^(e - 6) and more are what one call makes of them."""
    one, many = make_scaled([64], 2, 64, 32), make_scaled([64], 2, 64, 32)
    x = rand(64, 2, 64, dtype=torch.float32, seed=1) * torch.exp2(torch.arange(64) % 16 / 2).cuda()[:, None, None]
    one.append(x, -x, torch.tensor([64], dtype=torch.int32, device="cuda"))
    for i in range(64):
        many.append(x[i: i + 1], -x[i: i + 1], torch.tensor([i + 1], dtype=torch.int32, device="cuda"))
    assert torch.equal(one.scales.view(torch.uint8)[one.refs > 0], many.scales.view(torch.uint8)[many.refs > 0])
    a, b = values64(one)[0][one.refs > 0], values64(many)[0][many.refs > 0]
    e = torch.exp2(one.scales.view(torch.uint8).double() - 127 - 6).repeat_interleave(16, 3)[..., 0, None][one.refs > 0]
    assert torch.equal(torch.where(a.abs() >= e, a, 0.0), torch.where(a.abs() >= e, b, 0.0))
    assert float(((a - b).abs() / e).max()) <= 2.0 ** -3  # a step of the smallest numbers


def test_append_takes_strided_rows_and_leaves_out_those_without_pages():
    lens, rows = [40, 30, 20], [40, 9, 0]
    cache = make_scaled(lens, 2, 64, 16, seed=3)
    cache.table[0, 1], cache.table[1, 1] = -1, 1 << 20
    wide = rand(60, 5, 64, dtype=torch.bfloat16, seed=6)
    k, v = wide[:49, 0:2], wide[:49, 3:5]
    want = append64(cache, k, v, lens, rows)
    dl, off = rows_of(lens, rows, True)
    cache.append(wide[:, 0:2], wide[:, 3:5], dl, row_off=off)  # (11 rows more, which belong to nobody)
    same_pools(cache, *want)


# heads, KV heads, head dim, page, lens, rows
SHAPES = [(8, 8, 64, 16, [1], 1), (32, 8, 64, 16, [517], 1), (8, 2, 128, 32, [5, 300, 64, 17], 1), (4, 4, 32, 16, [700, 33], 5),
          (16, 2, 128, 64, [129, 64, 1000], 4), (8, 1, 64, 256, [2000, 1, 255], 8), (6, 2, 32, 32, [200, 90], 33),
          (8, 1, 128, 16, [150], 40), (16, 2, 64, 64, [300, 65], 0), (4, 2, 128, 16, [513, 40, 1], 0), (3, 1, 32, 128, [300], 0),
          (8, 8, 128, 64, [600, 450], -1), (1, 1, 128, 1024, [4000], 1)]


def rows_in(lens, rows):
    return [min(rows, n) for n in lens] if rows > 0 else list(lens) if rows == 0 else [1 + (n - 1) * (3 + i) // 9 for i, n in enumerate(lens)]


@pytest.mark.parametrize("dtype", list(T))
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (50, 4), (129, 17), (5000, 1)])
@pytest.mark.parametrize("clean", [False, True])
@pytest.mark.parametrize("h,hkv,hd,page,lens,rows", SHAPES, ids=str)
def test_attention(dtype, h, hkv, hd, page, lens, rows, window, sinks, clean):
    cache = make_scaled(lens, hkv, hd, page, layers=2, seed=hd + len(lens), clean=clean)
    rows = rows_in(lens, rows)
    q = rand(sum(rows), h, hd, dtype=T[dtype], seed=9)
    dl, off = rows_of(lens, rows, packed=min(rows) < max(rows))
    got = cache.attend(q, dl, layer=1, row_off=off, window=window or None, sinks=sinks)
    check(got, cache, q, lens, rows, layer=1, window=window, sinks=sinks)


@pytest.mark.parametrize("dtype", list(T))
@pytest.mark.parametrize("window,sinks", [(0, 0), (70, 3)])
@pytest.mark.parametrize("rows", [1, 3, 40, 90])
def test_attention_over_missing_pages_and_empty_rows(dtype, window, sinks, rows):
    lens = [100, 64, 40, 90, 300]
    cache = make_scaled(lens, 2, 64, 16, seed=1, clean=rows != 3)
    cache.table[0, 0:4] = -1
    cache.table[1, :] = -1           # a sequence without pages: zeros
    cache.table[2, 1] = cache.n_pages
    cache.table[3, 3:] = -1
    r = [min(rows, n) for n in lens]
    q = rand(sum(r), 8, 64, dtype=T[dtype], seed=2)
    dl, off = rows_of(lens, r, True)
    check(cache.attend(q, dl, row_off=off, window=window or None, sinks=sinks), cache, q, lens, r, window=window, sinks=sinks)


@pytest.mark.parametrize("dtype", list(T))
@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 2)])
@pytest.mark.parametrize("rows,g", [(1, 1), (4, 2), (16, 4), (70, 4)])
def test_nan_of_a_position_reaches_the_rows_that_read_it(dtype, window, sinks, rows, g):
    lens = [120, 100]
    cache = make_scaled(lens, 2, 64, 16, seed=8)
    for j in (1, 55, 90, 99, 118):
        for b, n in enumerate(lens):
            if j < n:
                page = int(cache.table[b, j // 16])
                pool = cache.v.view(torch.uint8)
                pool[page, 0, b, j % 16, 3 * b + j % 5] = 0x7f if j % 2 else 0xff
    q = rand(2 * rows, 2 * g, 64, dtype=T[dtype], seed=2)
    dl, _ = rows_of(lens, [rows, rows], False)
    got = cache.attend(q, dl, window=window or None, sinks=sinks)
    check(got, cache, q, lens, [rows, rows], window=window, sinks=sinks)


@pytest.mark.parametrize("dtype", list(T))
def test_scores_far_apart_and_scales_at_their_ends(dtype):
    """Scores that rise along the sequence; blocks whose values are tiny; scale 0 and negative."""
    cache = make_scaled([800], 2, 64, 64, seed=4)
    e = torch.full_like(cache.scales.view(torch.uint8), 127)
    e[..., 0] = 127 - 9
    e[..., 1] = 27
    e[int(cache.table[0, 3]), ..., 1] = 127
    cache.scales.view(torch.uint8).copy_(e)
    for rows in (1, 4, 60):
        q = rand(rows, 8, 64, dtype=T[dtype], seed=5, by=4.0)
        dl, _ = rows_of([800], [rows], False)
        for scale in (None, 0.0, -0.5):
            check(cache.attend(q, dl, scale=scale), cache, q, [800], [rows], scale=scale)


# records of the scales of 12, 16 and 2048 bytes
@pytest.mark.parametrize("hkv,page", [(3, 32), (4, 32), (64, 256)])
def test_pages_take_their_scales_along(hkv, page):
    """Forks, copies on writing, trims and compactions of a small pool against a list model."""
    layers = 2
    from paper_2511_09844_amd.paged import PagedCache
    cache = PagedCache.empty(14, page, layers, hkv, 32, 4, 5, dtype=torch.float8_e4m3fn)
    model = PageModel(14, page, 4, 5)
    history = [[] for _ in range(4)]  # k rows of every sequence
    g = torch.Generator().manual_seed(0)

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")

    def write(b, n):
        first = len(history[b])
        lo, hi = [0] * 4, [0] * 4
        lo[b], hi[b] = first, first + n
        granted = cache.reserve(ints(lo), ints(hi)).tolist()
        assert granted == model.reserve(lo, hi)
        assert granted[b] == first + n
        rows = [0] * 4
        rows[b] = n
        x = (torch.randn(n, hkv, 32, generator=g) * 2.0 ** int(torch.randint(-3, 6, (1,), generator=g))).cuda()
        lens = ints([len(h) + r for h, r in zip(history, rows)])
        off = ints([0] * (b + 1) + [n] * (4 - b))
        for l in range(layers):
            cache.append(x, x * (l + 1), lens, layer=l, row_off=off)
        history[b] += list(x)

    def look():
        assert cache.table.tolist() == model.table and cache.refs.tolist() == model.refs
        k, v = values64(cache)
        for b, rows in enumerate(history):
            for j, x in enumerate(rows):
                p = model.table[b][j // page]
                for l in range(layers):
                    for pool, by in ((k, 1), (v, l + 1)):
                        # off by the block's magnitude: half a step of the number, or of the smallest ones, twice
                        e = float(cache.scales[p, l, :, j % page // 16, 0 if by == 1 and pool is k else 1].double().max())
                        got = pool[p, l, :, j % page]
                        assert bool(((got - by * x.double()).abs() <= 2.0 ** -4 * by * x.double().abs() + 2.0 ** -9 * e).all())

    write(0, 37)
    look()
    cache.fork([0, 0], [1, 2])
    model.fork([0, 0], [1, 2])
    history[1], history[2] = list(history[0]), list(history[0])
    look()
    write(1, 5)
    write(2, 30)
    write(0, 1)
    look()
    cache.trim(ints([-1, 0]))
    model.trim([-1, 0])
    history[1] = []
    live = cache.compact()
    assert int(live) == model.compact()
    look()
    write(3, 20)
    look()
