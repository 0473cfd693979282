"""Packed calls of more sequences than a wave has lanes, over 8 bits and under windows: the kernels find the sequence of a row, a
unit or a tile among the first 64 at once, and behind them 64 at a time (rows that are appended: by a search from 64 on)."""
import pytest
import torch

from paged_ref import make_cache, rows_of
from paged_scaled_ref import append64, check, make_scaled

pytestmark = pytest.mark.gpu
T = {"bf16": torch.bfloat16, "f32": torch.float32}
COUNTS = [63, 64, 65, 150]
KINDS = [("8", "bf16", None, 0), ("8", "f32", None, 0), ("8", "bf16", 70, 3), ("8", "f32", 70, 3), ("bf16", "bf16", 70, 3), ("f32", "f32", 70, 3)]


def rand(*shape, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=g).to(dtype).cuda()


def some(count, most):
    """Rows of each sequence, up to `most`: the first, the last, and runs of others have none."""
    return [0 if b == 0 or b == count - 1 or b % 7 in (3, 4) or 60 <= b < 63 else 1 + (5 * b) % most for b in range(count)]


@pytest.mark.parametrize("dtype", list(T))
@pytest.mark.parametrize("count", COUNTS)
@pytest.mark.parametrize("most", [1, 5, 40])
def test_append(dtype, count, most):
    rows = some(count, most)
    lens = [r + (11 * b) % 37 for b, r in enumerate(rows)]
    cache = make_scaled(lens, 2, 32, 16, seed=count)
    n = sum(rows)
    k, v = (rand(n, 2, 32, dtype=T[dtype], seed=s) for s in (1, 2))
    pools, scales = append64(cache, k, v, lens, rows)
    dl, off = rows_of(lens, rows, True)
    cache.append(k, v, dl, row_off=off, max_rows=most)
    for got, want in zip((cache.k, cache.v), pools):
        got = got.double().cpu()
        assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(0), want.nan_to_num(0))
    assert torch.equal(cache.scales.view(torch.uint8).cpu(), scales)


@pytest.mark.parametrize("held,dtype,window,sinks", KINDS)
@pytest.mark.parametrize("count", COUNTS)
@pytest.mark.parametrize("hkv,most", [(1, 1), (2, 6), (1, 110)])  # 2, 12 and 220 query vectors: k_pdecode, the prompts' kernels
def test_attention(held, dtype, window, sinks, count, hkv, most):
    rows = some(count, most)
    # short sequences, and long ones among the first 64 and behind, whose keys are split; one that is empty
    lens = [r + (11 * b) % 37 + (2100 if b in (2, 41, 61, 62) or b in (64, 66, 127, 140) else 0) for b, r in enumerate(rows)]
    lens[0] = 0
    make = (lambda *a, **kw: make_scaled(*a, clean=True, **kw)) if held == "8" else lambda n, *a, **kw: make_cache(n, T[held], *a, **kw)
    cache = make(lens, hkv, 32, 64, seed=count)
    q = rand(sum(rows), 2 * hkv, 32, dtype=T[dtype], seed=3)
    dl, off = rows_of(lens, rows, True)
    for w, s in ((window, sinks), (window and 1500, sinks)):
        check(cache.attend(q, dl, row_off=off, max_rows=most, window=w, sinks=s), cache, q, lens, rows, window=w or 0, sinks=s)


@pytest.mark.parametrize("held,dtype,window,sinks", KINDS)
@pytest.mark.parametrize("rows", [1, 120])
def test_attention_of_equal_rows(held, dtype, window, sinks, rows):
    lens = [rows + (13 * b) % 50 + (1700 if b in (5, 70, 100) else 0) for b in range(101)]
    make = (lambda *a, **kw: make_scaled(*a, clean=True, **kw)) if held == "8" else lambda n, *a, **kw: make_cache(n, T[held], *a, **kw)
    cache = make(lens, 1, 32, 32, seed=4)
    q = rand(101 * rows, 2, 32, dtype=T[dtype], seed=5)
    dl, _ = rows_of(lens, [rows] * 101, False)
    check(cache.attend(q, dl, window=window, sinks=sinks), cache, q, lens, [rows] * 101, window=window or 0, sinks=sinks)
