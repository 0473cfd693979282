"""Plain float64 forms of the operators on caches of 8 bits and on windows, for the tests of paper_2511_09844_amd.paged."""
import math

import torch

from paged_ref import make_cache

LEAST, MOST = -100, 119


def power_of(a):
    """The least e with 448 * 2^e >= a, in LEAST .. MOST."""
    if a == 0:
        return LEAST
    e = math.ceil(math.log2(a / 448)) - 1 if a / 448 > 0 else LEAST
    e = max(e, -400)
    while 448.0 * 2.0 ** e < a:
        e += 1
    return min(max(e, LEAST), MOST)


def nearest(x):
    """e4m3 numbers nearest to float64 x, ties to even, at most 448; what is no finite number as NaN."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(2.0 ** -6, 1e300))) - 3)
    y = (torch.round(x / step) * step).clamp(-448.0, 448.0)
    return torch.where(torch.isfinite(x), y, torch.full_like(y, math.nan))


def values64(cache):
    """(k, v) in float64, whatever the cache holds them in."""
    if not cache.held8:
        return cache.k.double(), cache.v.double()
    e = cache.scales.view(torch.uint8).double() - 127
    by = torch.exp2(e).repeat_interleave(16, 3)
    return cache.k.double() * by[..., 0, None], cache.v.double() * by[..., 1, None]


def make_scaled(lens, hkv, hd, page, layers=1, spare=3, extra_entries=1, seed=0, device="cuda", clean=False):
    """A cache of 8 bits of random numbers and powers, pages in no order; every slot behind a sequence's last position
    and every other page holds NaN, and other pages' scales are 255.  Random numbers beyond 448 are NaN too, a few in ten
    thousand, unless clean."""
    from paper_2511_09844_amd.paged import PagedCache
    c = make_cache(lens, torch.float32, hkv, hd, page, layers, spare, extra_entries, seed, device=device)
    g = torch.Generator().manual_seed(seed + 1)
    e = torch.randint(-12, -6, (c.n_pages, layers, hkv, page // 16, 2), generator=g)
    e[..., 0] = e[..., 0].clamp(max=-8)
    scales = (e + 127).to(torch.uint8)
    scales[~torch.isin(torch.arange(c.n_pages), c.table.cpu())] = 255
    pools = [x.cpu() * 128 for x in (c.k, c.v)]
    pools = [(x.clamp(-448, 448) if clean else x).to(torch.float8_e4m3fn).to(device) for x in pools]
    return PagedCache(*pools, c.table, c.refs, scales=scales.to(device).view(torch.float8_e8m0fnu))


def append64(cache, k, v, lens, rows, layer=0):
    """What the pools and scales hold after an append, as float64 numbers, bytes of the scales and where anything was
    written; block by block of the definition."""
    pools = [cache.k.double().cpu(), cache.v.double().cpu()]
    scales, page = cache.scales.view(torch.uint8).cpu().clone(), cache.page_size
    table, at = cache.table.tolist(), 0
    for b, (n, r) in enumerate(zip(lens, rows)):
        p, end, i = n - r, n, at
        if p < 0:
            i, p = i - p, 0
        while p < end:
            m = min(end - p, 16 - p % 16)
            pg = table[b][p // page] if p // page < cache.max_pages else -1
            if 0 <= pg < cache.n_pages:
                blk, s0 = p % page // 16, p % page
                for h in range(cache.n_kv_heads):
                    for w, x in enumerate((k, v)):
                        new = x[i: i + m, h].double().cpu()
                        fin = new[torch.isfinite(new)]
                        e = power_of(float(fin.abs().max()) if fin.numel() else 0.0)
                        if p % 16:
                            was = min(max(int(scales[pg, layer, h, blk, w]) - 127, LEAST), MOST)
                            e = max(e, was)
                            if e > was:
                                old = pools[w][pg, layer, h, blk * 16: s0]
                                pools[w][pg, layer, h, blk * 16: s0] = nearest(old * 2.0 ** (was - e))
                        pools[w][pg, layer, h, s0: s0 + m] = nearest(new * 2.0 ** -e)
                        scales[pg, layer, h, blk, w] = e + 127
            p, i = p + m, i + m
        at += r
    return pools, scales


def reads(pos, j, window, sinks):
    """Whether rows at pos [n] read positions j [m], [n][m]."""
    back = pos[:, None] - j[None]
    seen = back >= 0
    return seen if not window else seen & ((back < window) | (j[None] < sinks))


def attend64(cache, q, lens, rows, layer=0, scale=None, window=0, sinks=0):
    """(out, sum of the weights times |v|, largest sum of magnitudes in a score), row by row of the definition.  Values that
    a row does not read do not enter it, whatever they are."""
    hd, page, g = cache.head_dim, cache.page_size, q.shape[1] // cache.n_kv_heads
    scale = 1.0 / math.sqrt(hd) if scale is None else scale
    k, v = values64(cache)
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    absv, spread, at, table = torch.zeros_like(out), 0.0, 0, cache.table.tolist()
    for b, (n, r) in enumerate(zip(lens, rows)):
        pos = [j for j in range(n) if j // page < cache.max_pages and 0 <= table[b][j // page] < cache.n_pages]
        if pos and r:
            pg = torch.tensor([table[b][j // page] for j in pos], device=q.device)
            pos = torch.tensor(pos, device=q.device)
            keys, vals = (x[pg, layer, :, pos % page].transpose(0, 1) for x in (k, v))  # [hkv][positions][hd]
            seen = reads(n - r + torch.arange(r, device=q.device), pos, window, sinks)
            for h in range(q.shape[1]):
                x, y, z = q[at: at + r, h].double(), keys[h // g], vals[h // g]
                s = (x @ y.T.contiguous()) * scale
                mag = (x.abs() @ y.abs().T.contiguous()) * abs(scale)
                mag = mag[seen & torch.isfinite(mag)]
                spread = max(spread, float(mag.max()) if mag.numel() else 0.0)
                w = torch.softmax(s.masked_fill(~seen, -math.inf), -1)
                w = torch.where(seen.any(-1, keepdim=True), w, torch.zeros_like(w))
                bad = ~torch.isfinite(z)
                out[at: at + r, h] = w @ z.masked_fill(bad, 0.0)
                absv[at: at + r, h] = w @ z.abs().masked_fill(bad, 0.0)
                for c in bad.any(1).nonzero()[:, 0].tolist():  # a position's infinities and NaN, to the rows that read it
                    mine = seen[:, c]
                    out[at: at + r, h] += torch.where(mine[:, None] & bad[c], w[:, c, None] * z[c], 0.0)
        at += r
    return out, absv, spread


def attend_bound(out, absv, spread, dtype, longest, hd):
    """How far a row may be off, elementwise.  Of 8 bits the cache's values are exact in bf16, and an fp32 row enters as three
    bf16 numbers (what they leave out is at most 2^-24 of it), so a score is a sum of up to 3 hd products, off by at most
    (3 hd + 3) 2^-24 times the sum of their magnitudes (spread); its exponential by that, 2 more steps of its own and
    one each of the scaling and the subtracted maximum (a step is 2^-23 of the argument, at most 2 spread); the sums
    over `longest` positions, of three products each, by (3 longest + 8) 2^-24 relative, above and below the fraction.
    bf16 besides: the weights rounded to it (half a step, 2^-8), and the output."""
    rel = 2 * ((3 * hd + 3) * 2.0 ** -24 * spread + 4 * 2.0 ** -23 * (2 * spread + 1)) + 2 * (3 * longest + 8) * 2.0 ** -24
    bound = rel * absv + 1e-30
    if dtype == torch.bfloat16:
        bound = bound + 2.0 ** -8 * absv + 2.0 ** -8 * (out.abs() + 2.0 ** -8 * absv)
    return bound


def check(got, cache, q, lens, rows, layer=0, scale=None, window=0, sinks=0):
    ref, absv, spread = attend64(cache, q, lens, rows, layer, scale, window, sinks)
    bound = attend_bound(ref.nan_to_num(0, 0, 0), absv, spread, q.dtype, max(list(lens) + [1]), cache.head_dim)
    got = got.double()
    fine = torch.isfinite(ref)
    assert torch.equal(torch.isnan(got), torch.isnan(ref)) and torch.equal(got[~fine].nan_to_num(7.0), ref[~fine].nan_to_num(7.0))
    off = torch.where(fine, (got - ref).abs() - bound, torch.zeros_like(bound))
    assert off.numel() == 0 or float(off.max()) <= 0, f"off by {float((got - ref).abs()[fine].max())}, {int((off > 0).sum())} of {off.numel()} beyond their bound"
