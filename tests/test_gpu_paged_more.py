"""What callers of the paged calls may do beside the plain case: hints that are far off, rows that are columns of wider
tensors, rows behind the last sequence, pools past 32 bits, calls that do not go through the native binding, two graphs of
one cache."""
import math

import pytest
import torch

from paged_ref import make_cache, rows_of
from paged_scaled_ref import append64, attend64, check, make_scaled, values64

pytestmark = pytest.mark.gpu
T = {"bf16": torch.bfloat16, "f32": torch.float32}
KINDS = [("bf16", "bf16"), ("f32", "f32"), ("8", "bf16"), ("8", "f32")]  # what the cache holds, the rows' type


def rand(*shape, dtype, seed, by=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * by).to(dtype).cuda()


def cache_of(held, lens, *a, **k):
    return make_scaled(lens, *a, clean=True, **k) if held == "8" else make_cache(lens, T[held], *a, **k)


@pytest.mark.parametrize("held,dtype", KINDS)
@pytest.mark.parametrize("window,sinks", [(None, 0), (300, 5)])
@pytest.mark.parametrize("max_len", [1, 64, 50000])
@pytest.mark.parametrize("rows", [1, 9, 100])
def test_expected_lengths_that_are_far_off(held, dtype, window, sinks, max_len, rows):
    lens = [2500, 3, 900]
    cache = cache_of(held, lens, 2, 64, 64, extra_entries=800, seed=1)
    r = [min(rows, n) for n in lens]
    q = rand(sum(r), 4, 64, dtype=T[dtype], seed=rows)
    dl, off = rows_of(lens, r, True)
    for most in (None, rows, 5000):
        got = cache.attend(q, dl, row_off=off, max_len=max_len, max_rows=most, window=window, sinks=sinks)
        check(got, cache, q, lens, r, window=window or 0, sinks=sinks)


@pytest.mark.parametrize("held,dtype", KINDS)
@pytest.mark.parametrize("window,sinks", [(None, 0), (30, 5)])
@pytest.mark.parametrize("rows", [1, 5, 90])
def test_columns_of_wider_tensors_and_rows_of_nobody(held, dtype, window, sinks, rows):
    lens = [200, 90]
    cache = cache_of(held, lens, 2, 64, 16, seed=2)
    n = 2 * rows
    wide = rand(n + 3, 3 * 4 * 64 + 64, dtype=T[dtype], seed=3)
    q, out = wide[:, : 4 * 64].unflatten(1, (4, 64)), wide[:, 8 * 64: 12 * 64].unflatten(1, (4, 64))
    before = wide.clone()
    dl, off = rows_of(lens, [rows, rows], True)
    got = cache.attend(q, dl, row_off=off, window=window, sinks=sinks, out=out)
    assert got.data_ptr() == out.data_ptr()
    check(out[:n], cache, q[:n].clone(), lens, [rows, rows], window=window or 0, sinks=sinks)
    before[:n, 8 * 64: 12 * 64] = wide[:n, 8 * 64: 12 * 64]
    assert torch.equal(before, wide)  # nothing else was written, the 3 rows behind the last sequence's neither


@pytest.mark.parametrize("dtype", list(T))
def test_pools_past_32_bits(dtype):
    """8 bits: k and v of 4.8 GB each, the sequence on their last pages."""
    from paper_2511_09844_amd.paged import PagedCache
    page, hkv, hd = 1024, 8, 128
    n_pages = (4 << 30) // (page * hkv * hd) + 600
    cache = PagedCache.empty(n_pages, page, 1, hkv, hd, 1, 4, dtype=torch.float8_e4m3fn)
    cache.table[0, :3] = torch.tensor([n_pages - 1, 1, n_pages - 2], dtype=torch.int32)
    cache.refs[[n_pages - 1, 1, n_pages - 2]] = 1
    lens = torch.tensor([2100], dtype=torch.int32, device="cuda")
    k, v = rand(2100, hkv, hd, dtype=T[dtype], seed=1), rand(2100, hkv, hd, dtype=T[dtype], seed=2)
    cache.append(k, v, lens)
    # against the same rows in a small pool
    small = PagedCache.empty(3, page, 1, hkv, hd, 1, 4, dtype=torch.float8_e4m3fn)
    small.table[0, :3] = torch.tensor([0, 1, 2], dtype=torch.int32)
    small.append(k, v, lens)
    for j, p in enumerate((n_pages - 1, 1, n_pages - 2)):
        m = min(page, 2100 - j * page)
        assert torch.equal(cache.k[p, :, :, :m].view(torch.uint8), small.k[j, :, :, :m].view(torch.uint8))
        assert torch.equal(cache.v[p, :, :, :m].view(torch.uint8), small.v[j, :, :, :m].view(torch.uint8))
        s = -(-m // 16)
        assert torch.equal(cache.scales[p, :, :, :s].view(torch.uint8), small.scales[j, :, :, :s].view(torch.uint8))
    for rows in (1, 7, 200):
        q = rand(rows, 16, hd, dtype=T[dtype], seed=rows)
        for window, sinks in ((None, 0), (700, 3)):
            a, b = (c.attend(q, lens, window=window, sinks=sinks) for c in (cache, small))
            assert torch.equal(a, b) and bool(torch.isfinite(a).all())
    check(b, small, q, [2100], [200], window=700, sinks=3)


@pytest.mark.parametrize("held,dtype", KINDS)
def test_the_long_way_gives_the_same(held, dtype, monkeypatch):
    """Calls whose arguments are not plain go through the checks in Python."""
    lens, rows = [300, 40, 17], [3, 3, 3]
    a, b = (cache_of(held, lens, 2, 64, 16, extra_entries=8, seed=4) for _ in range(2))
    monkeypatch.setattr(b, "_plain", lambda: False)
    q, k, v = (rand(9, h, 64, dtype=T[dtype], seed=i) for i, h in enumerate((4, 2, 2)))
    dl, off = rows_of(lens, rows, True)

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")

    for i in range(3):
        res = []
        for c in (a, b):
            c.append(k, v, dl, row_off=off)
            outs = [c.attend(q, dl), c.attend(q, dl, row_off=off, window=20, sinks=1), c.attend(q, dl, scale=0.25, max_len=300)]
            granted = c.reserve(ints([lens[0], 0, 0]), ints([lens[0] + 40, 0, 0]))
            c.fork([0], (1,))
            c.slide(dl, 100, sinks=17)
            outs += [granted, c.table.clone(), c.refs.clone(), c.k.view(torch.uint8).clone()]
            res.append(outs)
        assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(*res))
    from paper_2511_09844_amd import binding as B
    for c in (a, b):
        for f in (lambda: c.attend(q, dl, layer=1), lambda: c.attend(q[:, :3], dl), lambda: c.attend(q, dl[:2]), lambda: c.append(k, v[:, :1], dl),
                  lambda: c.attend(q, dl, max_rows=2), lambda: c.attend(q, dl, row_off=off[:2]), lambda: c.attend(q, dl, out=q), lambda: c.fork([0], [0]),
                  lambda: c.fork([0], [7]), lambda: c.reserve(dl, dl[:1]), lambda: c.attend(q.transpose(0, 1), dl), lambda: c.attend(q, dl, max_len=0),
                  lambda: c.attend(q, dl, scale=math.nan), lambda: c.slide(dl, 2 ** 31)):
            with pytest.raises(B.Sd2Error):
                f()
    with pytest.raises(B.Sd2Error):
        a.attend(q.clone().requires_grad_(), dl)


@pytest.mark.parametrize("held", ["bf16", "8"])
def test_two_graphs_of_one_cache(held):
    """A graph of single tokens and one of prompts over the same cache, replayed in turn: their workspaces are their own."""
    lens = [600, 450]
    cache = cache_of(held, lens, 2, 64, 32, seed=6)
    one, many = rand(2, 8, 64, dtype=torch.bfloat16, seed=1), rand(2 * 100, 8, 64, dtype=torch.bfloat16, seed=2)
    dl, _ = rows_of(lens, [1, 1], False)

    def calls(q):
        return [cache.attend(q, dl, window=w, sinks=s) for w, s in ((None, 0), (500, 3))]

    want = [[x.clone() for x in calls(q)] for q in (one, many)]
    graphs, outs = [], []
    for q in (one, many):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(calls(q))
        graphs.append(g)
    for i in range(6):
        for o in outs[i % 2]:
            o.zero_()
        graphs[i % 2].replay()
        if i % 3 == 0:
            torch.cuda.synchronize()
        junk = torch.full((1 << 22,), float("nan"), device="cuda")  # (eager memory between the replays)
        assert all(torch.equal(x, y) for x, y in zip(outs[i % 2], want[i % 2]))
        del junk


def test_a_block_fills_up_token_by_token_on_every_page_size():
    """One token at a time, its magnitude rising and falling, over the ends of blocks and pages."""
    for page in (16, 64):
        cache = make_scaled([1], 1, 32, page, extra_entries=70 // page + 1, spare=8, seed=page)
        free = [p for p in range(cache.n_pages) if p not in cache.table[0].tolist()]
        cache.table[0] = torch.tensor([int(cache.table[0, 0])] + free[: cache.max_pages - 1], dtype=torch.int32)
        g = torch.Generator().manual_seed(page)
        for n in range(1, 70):
            x = (torch.randn(1, 1, 32, generator=g) * 2.0 ** float(torch.randint(-9, 10, (1,), generator=g))).cuda()
            y = x.flip(2) * (0.0 if n % 7 == 0 else 1.0)
            want = append64(cache, x, y, [n], [1])
            cache.append(x, y, torch.tensor([n], dtype=torch.int32, device="cuda"))
            for got, ref in zip((cache.k, cache.v), want[0]):
                got = got.double().cpu()
                assert torch.equal(got.isnan(), ref.isnan()) and torch.equal(got.nan_to_num(0), ref.nan_to_num(0))
            assert torch.equal(cache.scales.view(torch.uint8).cpu(), want[1])
        assert bool(torch.isfinite(values64(cache)[0][cache.table[0].long()].flatten(1)[0]).all())
