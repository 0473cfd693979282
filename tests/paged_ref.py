"""Plain float64 attention over a paged cache and a list model of its pages, for the tests of
paper_2511_09844_amd.paged."""
import math

import torch


def make_cache(lens, dtype, hkv, hd, page, layers=1, spare=3, extra_entries=1, seed=0, stale=float("nan"), device="cuda"):
    """A PagedCache whose sequences hold lens positions of N(0, 1) rows on pages in no order; every slot
    behind a sequence's last position and every other page holds `stale`."""
    from paper_2511_09844_amd.paged import PagedCache
    g = torch.Generator().manual_seed(seed)
    used = [-(-n // page) for n in lens]
    n_pages = sum(used) + spare
    shape = (n_pages, layers, hkv, page, hd)
    k, v = torch.randn(shape, generator=g).to(dtype), torch.randn(shape, generator=g).to(dtype)
    order = torch.randperm(n_pages, generator=g).tolist()
    table = torch.full((len(lens), max(used + [0]) + extra_entries), -1, dtype=torch.int32)
    refs = torch.zeros(n_pages, dtype=torch.int32)
    at, live = 0, torch.zeros(n_pages, page, dtype=torch.bool)
    for b, n in enumerate(lens):
        for j in range(used[b]):
            p = order[at]
            at += 1
            table[b, j] = p
            refs[p] = 1
            live[p, : min(page, n - j * page)] = True
    for pool in (k, v):
        pool.transpose(1, 3)[~live] = stale  # [n_pages][page] first
    return PagedCache(k.to(device), v.to(device), table.to(device), refs.to(device))


def rows_of(lens, rows, packed, device="cuda"):
    """(lens, row_off or None) as device tensors."""
    off = [sum(rows[:i]) for i in range(len(rows) + 1)]
    return (torch.tensor(lens, dtype=torch.int32, device=device),
            torch.tensor(off, dtype=torch.int32, device=device) if packed else None)


def attend64(cache, q, lens, rows, layer=0, scale=None):
    """(out, sum of the weights times |v|, largest |score|) in float64, row by row of the definition."""
    hd, page, g = cache.head_dim, cache.page_size, q.shape[1] // cache.n_kv_heads
    scale = 1.0 / math.sqrt(hd) if scale is None else scale
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    absv = torch.zeros_like(out)
    spread = 0.0
    at = 0
    table = cache.table.tolist()
    for b, (n, r) in enumerate(zip(lens, rows)):
        pos = [j for j in range(n) if j // page < cache.max_pages and 0 <= table[b][j // page] < cache.n_pages]
        if pos and r:
            pg = torch.tensor([table[b][j // page] for j in pos], device=q.device)
            sl = torch.tensor([j % page for j in pos], device=q.device)
            keys = cache.k[pg, layer, :, sl].double()      # [positions][hkv][hd]
            vals = cache.v[pg, layer, :, sl].double()
            mine = n - r + torch.arange(r, device=q.device)
            seen = torch.tensor(pos, device=q.device)[None] <= mine[:, None]
            for h in range(q.shape[1]):
                s = (q[at: at + r, h].double() @ keys[:, h // g].T.contiguous()) * scale
                spread = max(spread, float(torch.where(seen, (q[at: at + r, h].double().abs() @ keys[:, h // g].abs().T.contiguous())
                                                       * abs(scale), torch.zeros_like(s)).max()))
                s = s.masked_fill(~seen, -math.inf)
                w = torch.softmax(s, -1)
                w = torch.where(seen.any(-1, keepdim=True), w, torch.zeros_like(w))
                out[at: at + r, h] = w @ vals[:, h // g]
                absv[at: at + r, h] = w @ vals[:, h // g].abs()
        at += r
    return out, absv, spread


def attend_bound(out, absv, spread, dtype, longest, hd):
    """How far a row may be off, elementwise.  A score's fp32 sum of hd products is off by at most
    (hd + 2) 2^-24 times the sum of their magnitudes (spread), its exponential by that, 2 more steps of
    its own and one each of the scaling and the subtracted maximum (a step is 2^-23 of the argument, which
    is at most 2 spread); the sums over `longest` positions by (longest + 8) 2^-24 relative, above and below the
    fraction.  bf16 besides: the weights rounded to it (half a step, 2^-8), and the output."""
    rel = 2 * ((hd + 2) * 2.0 ** -24 * spread + 4 * 2.0 ** -23 * (2 * spread + 1)) + 2 * (longest + 8) * 2.0 ** -24
    bound = rel * absv + 1e-30
    if dtype == torch.bfloat16:
        bound = bound + 2.0 ** -8 * absv + 2.0 ** -8 * (out.abs() + 2.0 ** -8 * absv)
    return bound


class PageModel:
    """The book-keeping of a cache on lists: which row of data every slot holds goes along as tags."""

    def __init__(self, n_pages, page, seqs, entries):
        self.page, self.refs = page, [0] * n_pages
        self.table = [[-1] * entries for _ in range(seqs)]
        self.tags = [[None] * page for _ in range(n_pages)]

    def reserve(self, first, last, keep=None):
        keep = first if keep is None else keep
        free, before, granted = [p for p, r in enumerate(self.refs) if r == 0], list(self.refs), []
        for b, (lo, hi, kp) in enumerate(zip(first, last, keep)):
            lo, hi, kp = max(lo, 0), max(hi, 0), max(kp, 0)
            end = min(hi, len(self.table[b]) * self.page)
            for j in range(len(self.table[b])):
                if not (lo < hi and lo // self.page <= j and j * self.page < hi):
                    continue
                p = self.table[b][j]
                if p >= 0 and before[p] <= 1:
                    continue
                if not free:
                    end = min(end, j * self.page)
                    continue
                new = free.pop(0)
                if p >= 0:
                    n = max(0, min(self.page, kp - j * self.page))
                    self.tags[new][:n] = self.tags[p][:n]
                    self.refs[p] -= 1
                self.refs[new] = 1
                self.table[b][j] = new
            granted.append(end)
        return granted

    def fork(self, src, dst):
        for s, d in zip(src, dst):
            old = self.table[d]
            self.table[d] = list(self.table[s])
            for p in self.table[d]:
                if p >= 0:
                    self.refs[p] += 1
            for p in old:
                if p >= 0:
                    self.refs[p] -= 1

    def trim(self, lens):
        for b, n in enumerate(lens):
            if n < 0:
                continue
            for j in range(-(-n // self.page), len(self.table[b])):
                if self.table[b][j] >= 0:
                    self.refs[self.table[b][j]] -= 1
                    self.table[b][j] = -1

    def compact(self):
        live = sum(r > 0 for r in self.refs)
        holes = [p for p in range(live) if self.refs[p] == 0]
        for p in range(live, len(self.refs)):
            if self.refs[p] > 0:
                to = holes.pop(0)
                self.tags[to], self.refs[to], self.refs[p] = list(self.tags[p]), self.refs[p], 0
                self.table = [[to if x == p else x for x in row] for row in self.table]
        return live
