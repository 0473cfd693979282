"""How exactly the softmax's weights enter the product with V where bf16 rows are few: as two bf16 numbers each, off by at most
2^-15, not as one, off by 2^-8.  V is 1 or -1 (of the longest sequence at every 16th position, elsewhere 0) and the weights nearly equal, so
that the outputs, and with them their own rounding, are far smaller than the sum of such errors may be."""
import pytest
import torch

from paged_ref import make_cache, rows_of
from paged_scaled_ref import attend64, attend_bound, make_scaled

BF16 = torch.bfloat16
LENS = [2, 3, 9, 48, 700]
HD = 64


def rows_q(n):
    return (torch.randn(n, 8, HD, generator=torch.Generator().manual_seed(2)) * 0.2).to(BF16)


def signs(shape):
    return torch.where(torch.rand(shape, generator=torch.Generator().manual_seed(1)) < 0.5, -1.0, 1.0)


def bound_of(ref, absv, spread):
    """attend_bound for fp32 (scores, exponentials, sums); the leading digits of a weight are off by less than 2^-7 of it, and what
    they leave out is rounded, 2^-8 of that; the output's rounding."""
    b = attend_bound(ref, absv, spread, torch.float32, max(LENS), HD) + 2.0 ** -15 * absv
    return b + 2.0 ** -8 * (ref.abs() + b)


@pytest.mark.gpu
@pytest.mark.parametrize("held,window,sinks", [("8", 0, 0), ("8", 600, 1), ("bf16", 0, 0), ("bf16", 600, 1)])
@pytest.mark.parametrize("rows", [1, 4, 5, 16])  # 4 to 64 query vectors of a KV head
@pytest.mark.parametrize("entries", [1, 400])    # one unit for a sequence; units that are joined
def test_few_bf16_rows(held, window, sinks, rows, entries):
    if held == "8":
        cache = make_scaled(LENS, 2, HD, 16, extra_entries=entries, seed=3, clean=True)
        scales = cache.scales.view(torch.uint8)
        scales[..., 0], scales[..., 1] = 127 - 7, 127
    else:
        cache = make_cache(LENS, BF16, 2, HD, 16, extra_entries=entries, seed=3)
    v = signs(cache.v.shape)
    for p in cache.table[-1].tolist():
        if p >= 0:
            v[p, :, :, torch.arange(16) != 5] = 0.0
    cache.v.copy_(v.to(cache.v.dtype))
    r = [min(rows, n) for n in LENS]
    q = rows_q(sum(r)).cuda()
    dl, off = rows_of(LENS, r, True)
    ref, absv, spread = attend64(cache, q, LENS, r, window=window, sinks=sinks)
    got = cache.attend(q, dl, row_off=off, max_rows=rows, window=window or None, sinks=sinks).double()
    beyond = float(((got - ref).abs() / bound_of(ref, absv, spread)).max())
    assert beyond <= 1, f"{beyond} of the bound"


@pytest.mark.parametrize("part", ["leading digits", "rounded once"])
def test_the_bound_notices_weights_of_one_number(part):
    q = rows_q(40).double()
    for n in LENS:
        g = torch.Generator().manual_seed(n)
        k, v = torch.randn(n, HD, generator=g).double(), signs((n, HD)).double()
        if n == LENS[-1]:
            v[torch.arange(n) % 16 != 5] = 0.0
        w = torch.softmax((q @ k.T) / 8, -1)
        spread = float((q.abs() @ k.abs().T).max()) / 8
        x = w / w.amax(-1, keepdim=True)  # (as they are summed: the largest is 1)
        if part == "rounded once":
            y = x.to(BF16).double()
        else:
            y = ((x.float().view(torch.int32) - 1) & -65536).view(torch.float32).double()
        ref, got = w @ v, (y @ v) / x.sum(-1, keepdim=True)
        assert float(((got - ref).abs() / bound_of(ref, w @ v.abs(), spread)).max()) > 1, n
