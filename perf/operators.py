"""The paged K/V cache's operators as cases that can be timed and compared.

A cache of pages: k and v are pools [n_pages][layers][kv heads][page][head dim]; row b of the table
names the pages of sequence b in the order of its positions (-1: none); refs counts for every page the
table entries that name it.  Four operators work on it:

  attend   attention of each sequence's newest rows over its pages, causal, with grouped heads: one row
           (decoding), the rows of a speculative block, or whole prompts packed one after another
  append   new K/V rows into the pages
  fork     sequences that go on from another one's pages, and the pages they then write to: shared ones
           are copied (fork and reserve)
  move     a sequence copied page by page, its original freed, what is left moved together (fork,
           reserve, trim, compact), and the sequence put back under its first name

Pages lie in the pool in no order, as after many requests, and hold old values behind the last row.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _attend(name, dtype, h, hkv, hd, page, seqs, lo, hi, rows):
    c = {"op": "attend", "dtype": dtype, "h": h, "hkv": hkv, "hd": hd, "page": page, "seqs": seqs, "lo": lo, "hi": hi,
         "rows": rows}
    return dict(c, name=name) if name else c


def _append(name, dtype, hkv, hd, page, layers, seqs, lo, hi, rows):
    c = {"op": "append", "dtype": dtype, "hkv": hkv, "hd": hd, "page": page, "layers": layers, "seqs": seqs, "lo": lo,
         "hi": hi, "rows": rows}
    return dict(c, name=name) if name else c


def _pages(name, op, dtype, hkv, hd, page, layers, n_pages, seqs, hi):
    c = {"op": op, "dtype": dtype, "hkv": hkv, "hd": hd, "page": page, "layers": layers, "n_pages": n_pages,
         "seqs": seqs, "hi": hi}
    return dict(c, name=name) if name else c


def listed():
    # rows: how many each sequence brings; 0: all its positions (a prompt); -1: a different part of them for
    # each (chunks of prompts over what is cached already)
    return [
        # a drafter's step for one user: the smallest call, latency counts
        _attend("decode-1", "bf16", 32, 8, 64, 16, 1, 517, 517, 1),
        # a verifier-shaped decoding step of 16 ragged sequences, fp32 caches
        _attend("decode-16-f32", "f32", 32, 8, 128, 32, 16, 256, 2048, 1),
        # two long documents, an odd length
        _attend("decode-long", "bf16", 32, 8, 128, 64, 2, 90001, 131071, 1),
        # the verify pass of a speculative block (k = 7) for 16 ragged sequences, the engine's fp32 caches
        _attend("verify-16-f32", "f32", 32, 8, 128, 32, 16, 256, 2048, 8),
        # one long prompt
        _attend("prompt-8192", "bf16", 32, 8, 128, 64, 1, 8192, 8192, 0),
        # prompts that arrive together, from one token up
        _attend("prompts-packed", "bf16", 32, 8, 128, 64, 24, 1, 2001, 0),
        # chunks of prompts over what is cached, one query head per KV head, fp32
        _attend("chunks-f32", "f32", 12, 12, 64, 16, 5, 97, 1290, -1),
        # one token of 16 sequences into one layer's pages
        _append("append-16", "f32", 8, 128, 32, 4, 16, 256, 2048, 1),
        # a prompt's rows into one layer's pages
        _append("append-prompts", "bf16", 8, 128, 64, 4, 8, 1000, 8191, 0),
        # four samples of one short prompt on a small model
        _pages("fork-4", "fork", "f32", 8, 32, 16, 4, 64, 4, 45),
        # 32 samples of one prompt on an 8B-sized verifier's cache
        _pages("fork-32", "fork", "bf16", 8, 128, 64, 32, 160, 32, 2011),
        # a long sequence copied and moved together, 8B-sized
        _pages("move-5000", "move", "bf16", 8, 128, 64, 32, 240, 3, 5000),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5))))))


def draw(rng):
    op = rng.choice(["decode", "decode", "verify", "prompt", "prompt", "chunk", "append", "fork", "move"])
    dtype, hd, page = rng.choice(["bf16", "f32"]), rng.choice([32, 64, 128]), rng.choice([16, 32, 64, 128, 256])
    hkv = rng.choice([1, 2, 4, 8, 12])
    h = hkv * rng.choice([1, 2, 3, 4, 8])
    layers = rng.choice([1, 2, 3, 8])
    seqs = _log_int(rng, 1, 40)
    if op == "decode":
        hi = _log_int(rng, 1, 160000 // seqs)
        return _attend(None, dtype, h, hkv, hd, page, seqs, _log_int(rng, 1, hi), hi, 1)
    if op == "verify":
        rows = rng.randint(2, 33)
        hi = _log_int(rng, rows, max(rows, 40000 // seqs))
        return _attend(None, dtype, h, hkv, hd, page, seqs, _log_int(rng, rows, hi), hi, rows)
    if op in ("prompt", "chunk"):
        hi = _log_int(rng, 2, 4000 if dtype == "bf16" else 2000)
        seqs = _log_int(rng, 1, max(1, 6000 // hi))
        return _attend(None, dtype, h, hkv, hd, page, seqs, _log_int(rng, 1, hi), hi, 0 if op == "prompt" else -1)
    if op == "append":
        hi = _log_int(rng, 1, 40000 // seqs)
        return _append(None, dtype, hkv, hd, page, layers, seqs, _log_int(rng, 1, hi), hi, rng.choice([1, 0, -1]))
    hi = _log_int(rng, 1, 4000)
    used = -(-hi // page)
    if op == "fork":
        seqs = _log_int(rng, 2, 32)
        return _pages(None, op, dtype, hkv, hd, page, layers, used + 2 * seqs + rng.randint(2, 40), seqs, hi)
    return _pages(None, op, dtype, hkv, hd, page, layers, 2 * used + rng.randint(2, 40), 3, hi)


# ---- shapes ------------------------------------------------------------------------------------

def _lens(case):
    """Lengths of the sequences, spread evenly over the range, the longest one first."""
    n, lo, hi = case["seqs"], case["lo"], case["hi"]
    return [hi - (hi - lo) * i // max(1, n - 1) for i in range(n)]


def _rows(case):
    """How many of its last positions each sequence brings."""
    lens = _lens(case)
    if case["rows"] > 0:
        return [min(case["rows"], n) for n in lens]
    return [n if case["rows"] == 0 else 1 + (n - 1) * ((7 * i + 3) % 10) // 10 for i, n in enumerate(lens)]


def _row_bytes(case):
    return case["hd"] * (2 if case["dtype"] == "bf16" else 4)


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "attend":
        lens, rows = _lens(case), _rows(case)
        pairs = sum(n * r - r * (r - 1) // 2 for n, r in zip(lens, rows))
        kv, qo = 2 * sum(lens) * case["hkv"] * case["hd"] * size, 2 * sum(rows) * case["h"] * case["hd"] * size
        return {"bytes": kv + qo, "flops": 4.0 * pairs * case["h"] * case["hd"]}
    if case["op"] == "append":
        return {"bytes": 4.0 * sum(_rows(case)) * case["hkv"] * _row_bytes(case), "flops": 0}
    table = 4.0 * (case["n_pages"] + case["seqs"] * -(-case["hi"] // case["page"]))
    row = 2 * case["layers"] * case["hkv"] * _row_bytes(case)  # a position of k and v in all layers
    if case["op"] == "fork":
        # the copies' part of the last page, when it is shared
        return {"bytes": table + 2.0 * row * (case["seqs"] - 1) * (case["hi"] % case["page"]), "flops": 0}
    # copied once when it is written to, and its pages once more when they are moved together
    used = -(-case["hi"] // case["page"])
    return {"bytes": table + 2.0 * row * (case["hi"] + used * case["page"]), "flops": 0}


# ---- inputs --------------------------------------------------------------------------------------

def _cache(case, gen, layers, n_pages, lens):
    """Pools of old values, and a table whose sequences hold lens positions on pages in no order."""
    shape = (n_pages, layers, case["hkv"], case["page"], case["hd"])
    dt = TYPES[case["dtype"]]
    k = torch.empty(shape, dtype=dt, device="cuda").normal_(0.0, 1.0, generator=gen)
    v = torch.empty(shape, dtype=dt, device="cuda").normal_(0.0, 1.0, generator=gen)
    used = [-(-n // case["page"]) for n in lens]
    table = torch.full((len(lens), max(1, -(-case["hi"] // case["page"])) + 1), -1, dtype=torch.int32)
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(gen.initial_seed())).to(torch.int32)
    at = 0
    for b, n in enumerate(used):
        table[b, :n] = order[at: at + n]
        at += n
    refs = torch.zeros(n_pages, dtype=torch.int32)
    refs[order[:at].long()] = 1
    return {"k": k, "v": v, "table": table.cuda(), "refs": refs.cuda()}


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed * 7919 + 17)
    dt = TYPES[case["dtype"]]

    def randn(*shape):
        return torch.empty(shape, dtype=dt, device="cuda").normal_(0.0, 1.0, generator=gen)

    def ints(v):
        return torch.tensor(v, dtype=torch.int32).cuda()

    st = {"case": case}
    if case["op"] in ("attend", "append"):
        lens, rows = _lens(case), _rows(case)
        pages = sum(-(-n // case["page"]) for n in lens)
        layers = case.get("layers", 1)
        st.update(_cache(case, gen, layers, pages + 3, lens))
        st["layer"] = layers - 1
        st["lens"] = ints(lens)
        st["most"], st["max_len"], st["total"] = max(rows), max(lens), sum(rows)
        # the first row of every sequence, and behind the last one their number; none where all bring the same
        st["row_off"] = None
        if min(rows) < max(rows):
            st["row_off"] = ints([sum(rows[:i]) for i in range(len(rows) + 1)])
        if case["op"] == "attend":
            st["q"] = randn(sum(rows), case["h"], case["hd"])
        else:
            st["new_k"], st["new_v"] = randn(sum(rows), case["hkv"], case["hd"]), randn(sum(rows), case["hkv"], case["hd"])
    else:
        lens = [case["hi"]] + [0] * (case["seqs"] - 1)
        st.update(_cache(case, gen, case["layers"], case["n_pages"], lens))
        n = case["seqs"]
        if case["op"] == "fork":
            # the copies write their next 8 positions; the first sequence waits
            st["first"] = ints([case["hi"]] * n)
            st["last"] = ints([0] + [case["hi"] + 8] * (n - 1))
        else:
            # sequence 1 is to have every position on pages of its own
            st["first"], st["last"] = ints([0, 0, 0]), ints([0, case["hi"], 0])
            st["drop0"], st["drop1"] = ints([0, -1, -1]), ints([-1, 0, -1])
    if own:
        from paper_2511_09844_amd.paged import PagedCache
        st["cache"] = PagedCache(st["k"], st["v"], st["table"], st["refs"])
    return st


# ---- the plain form --------------------------------------------------------------------------------

def _row_index(st):
    """[sequences][most] index of every row, and whether there is one; their positions."""
    n = st["lens"].numel()
    i = torch.arange(st["most"], device="cuda")
    if st["row_off"] is None:
        start = torch.arange(n, device="cuda") * st["most"]
        rows = torch.full((n,), st["most"], device="cuda")
    else:
        start, rows = st["row_off"][:-1].long(), (st["row_off"][1:] - st["row_off"][:-1]).long()
    there = i[None] < rows[:, None]
    idx = torch.where(there, start[:, None] + i[None], 0)
    return idx, there, (st["lens"].long() - rows)[:, None] + i[None]


def _plain_attend(st):
    c = st["case"]
    page, hkv, hd, g = c["page"], c["hkv"], c["hd"], c["h"] // c["hkv"]
    n, most, length = c["seqs"], st["most"], st["max_len"]
    idx, there, pos = _row_index(st)
    entries = st["table"][:, : -(-length // page)].long().clamp(min=0)
    held = torch.arange(length, device="cuda")[None] < st["lens"][:, None]

    def rows_of(pool):
        x = pool[entries, st["layer"]].float()                      # [n][pages][hkv][page][hd]
        x = x.permute(0, 2, 1, 3, 4).reshape(n, hkv, -1, hd)[:, :, :length]
        return torch.where(held[:, None, :, None], x, torch.zeros((), device="cuda")).contiguous()

    q = st["q"][idx].float().view(n, most, hkv, g, hd).permute(0, 2, 3, 1, 4).reshape(n, hkv, g * most, hd)
    s = torch.matmul(q.contiguous(), rows_of(st["k"]).transpose(2, 3).contiguous()).view(n, hkv, g, most, length)
    s.mul_(1.0 / math.sqrt(hd))
    read = held[:, None, :] & (torch.arange(length, device="cuda") <= pos[:, :, None])
    s.masked_fill_(~read[:, None, None], -math.inf)
    s.sub_(s.amax(-1, keepdim=True)).exp_()
    total = s.sum(-1, keepdim=True)
    o = torch.matmul(s.view(n, hkv, g * most, length), rows_of(st["v"])).view(n, hkv, g, most, hd) / total
    o = o.permute(0, 3, 1, 2, 4).reshape(n, most, c["h"], hd)
    out = torch.empty_like(st["q"])
    out[idx[there]] = o[there].to(out.dtype)
    return out


def _plain_append(st):
    page = st["case"]["page"]
    idx, there, pos = _row_index(st)
    seq = torch.arange(pos.shape[0], device="cuda")[:, None].expand_as(pos)[there]
    at = pos[there]
    page_of = st["table"][seq, at // page].long()
    st["k"][page_of, st["layer"], :, at % page] = st["new_k"][idx[there]]
    st["v"][page_of, st["layer"], :, at % page] = st["new_v"][idx[there]]
    return {"k": st["k"], "v": st["v"]}


def _plain_fork(st, src, dst):
    table, refs = st["table"], st["refs"]
    for row, by in ((dst, -1), (src, 1)):
        entries = table[row].flatten()
        refs.index_add_(0, entries.clamp(min=0).long(), torch.where(entries >= 0, by, 0).to(torch.int32))
    table[dst] = table[src]


def _plain_reserve(st, first, last, keep):
    """Pages for positions first .. last - 1 of every sequence that no other one shares; of a shared one
    the positions below keep are copied."""
    table, refs, page = st["table"], st["refs"], st["case"]["page"]
    j = torch.arange(table.shape[1], device="cuda")[None]
    first, last, keep = first[:, None].long(), last[:, None].long(), keep[:, None].long()
    window = (j >= first // page) & (j * page < last) & (first < last)
    entry = table.long()
    shared = window & (entry >= 0) & (refs[entry.clamp(min=0)] > 1)
    need = window & ((entry < 0) | shared)
    free = (refs == 0).nonzero()[:, 0]
    rank = (need.flatten().cumsum(0) - 1).view_as(need)
    got = need & (rank < free.numel())
    new = free[rank[got]]
    copy = shared & got
    src, dst = entry[copy], free[rank[copy]]
    kept = (keep - j * page).clamp(0, page)[copy]
    slot = (torch.arange(page, device="cuda")[None] < kept[:, None])[:, None, None, :, None]
    for pool in (st["k"], st["v"]):
        pool[dst] = torch.where(slot, pool[src], pool[dst])
    refs.index_add_(0, src, torch.full_like(src, -1, dtype=torch.int32))
    refs[new] = 1
    table[got] = new.to(torch.int32)
    bad = need & ~got
    lead = torch.where(bad, j, table.shape[1]).amin(1)
    return torch.minimum(last[:, 0].clamp(min=0), lead * page).to(torch.int32)


def _plain_trim(st, lens):
    table, refs, page = st["table"], st["refs"], st["case"]["page"]
    j = torch.arange(table.shape[1], device="cuda")[None]
    drop = (lens[:, None] >= 0) & (j * page >= lens[:, None]) & (table >= 0)
    refs.index_add_(0, table[drop].long(), torch.full_like(table[drop], -1))
    table[drop] = -1


def _plain_compact(st):
    table, refs = st["table"], st["refs"]
    live = refs > 0
    count = live.sum()
    at = torch.arange(refs.numel(), device="cuda")
    src, dst = at[live & (at >= count)], at[~live & (at < count)]
    for pool in (st["k"], st["v"]):
        pool[dst] = pool[src]
    refs[dst], refs[src] = refs[src], 0
    name = at.clone()
    name[src] = dst
    table.copy_(torch.where(table >= 0, name[table.clamp(min=0).long()].to(torch.int32), table))
    return count.to(torch.int32)[None]


def _plain(st):
    op = st["case"]["op"]
    if op == "attend":
        return _plain_attend(st)
    if op == "append":
        return _plain_append(st)
    out = {"k": st["k"], "v": st["v"], "table": st["table"], "refs": st["refs"]}
    if op == "fork":
        n = st["case"]["seqs"]
        _plain_fork(st, [0] * (n - 1), list(range(1, n)))
        return dict(out, granted=_plain_reserve(st, st["first"], st["last"], st["first"]))
    _plain_fork(st, [0], [1])
    granted = _plain_reserve(st, st["first"], st["last"], st["last"])
    _plain_trim(st, st["drop0"])
    live = _plain_compact(st)
    _plain_fork(st, [1], [0])
    _plain_trim(st, st["drop1"])
    return dict(out, granted=granted, live=live)


# ---- the framework's calls ---------------------------------------------------------------------------

def _own(st):
    op, cache = st["case"]["op"], st["cache"]
    if op == "attend":
        return cache.attend(st["q"], st["lens"], layer=st["layer"], row_off=st["row_off"], max_rows=st["most"],
                            max_len=st["max_len"])
    if op == "append":
        cache.append(st["new_k"], st["new_v"], st["lens"], layer=st["layer"], row_off=st["row_off"], max_rows=st["most"])
        return {"k": cache.k, "v": cache.v}
    out = {"k": cache.k, "v": cache.v, "table": cache.table, "refs": cache.refs}
    if op == "fork":
        n = st["case"]["seqs"]
        cache.fork([0] * (n - 1), list(range(1, n)))
        return dict(out, granted=cache.reserve(st["first"], st["last"]))
    cache.fork([0], [1])
    granted = cache.reserve(st["first"], st["last"], keep=st["last"])
    cache.trim(st["drop0"])
    live = cache.compact()
    cache.fork([1], [0])
    cache.trim(st["drop1"])
    return dict(out, granted=granted, live=live)


def run(state):
    return _own(state) if own else _plain(state)


# ---- the same in 64 bits, sequence by sequence -----------------------------------------------------------

def _exact_attend(case, st):
    lens, rows, page, hd = _lens(case), _rows(case), case["page"], case["hd"]
    g, out, at = case["h"] // case["hkv"], torch.empty(st["q"].shape, dtype=torch.float64, device="cuda"), 0
    for b, (n, r) in enumerate(zip(lens, rows)):
        pages = st["table"][b, : -(-n // page)].tolist()
        for head in range(case["hkv"]):
            keys, values = (torch.cat([pool[p, 0, head] for p in pages])[:n].double() for pool in (st["k"], st["v"]))
            for i in range(0, r, 2048):
                m = min(2048, r - i)
                qs = st["q"][at + i: at + i + m, head * g: (head + 1) * g].double().transpose(0, 1).reshape(g * m, hd)
                seen = n - r + i + m
                score = (qs @ keys[:seen].T.contiguous() / math.sqrt(hd)).view(g, m, seen)
                later = torch.ones(m, seen, dtype=torch.bool, device="cuda").triu(n - r + i + 1)
                weight = torch.softmax(score.masked_fill(later, -math.inf), dim=-1).view(g * m, seen)
                res = (weight @ values[:seen]).view(g, m, hd)
                out[at + i: at + i + m, head * g: (head + 1) * g] = res.transpose(0, 1)
        at += r
    return out


def _exact_append(case, st):
    page, layer = case["page"], case["layers"] - 1
    pools, at = {"k": st["k"].double(), "v": st["v"].double()}, 0
    for b, (n, r) in enumerate(zip(_lens(case), _rows(case))):
        pages = st["table"][b].tolist()
        p = n - r
        while p < n:  # from one page to the next
            m = min(n - p, page - p % page)
            for name in ("k", "v"):
                rows = st["new_" + name][at: at + m].double().transpose(0, 1)
                pools[name][pages[p // page], layer, :, p % page: p % page + m] = rows
            p, at = p + m, at + m
    return pools


def _exact_pages(case, st):
    """The same steps on lists, a page and a sequence at a time."""
    page, k, v = case["page"], st["k"].double(), st["v"].double()
    table, refs = st["table"].tolist(), st["refs"].tolist()

    def move(src, dst, slots):
        for pool in (k, v):
            pool[dst, :, :, :slots] = pool[src, :, :, :slots]

    def drop(b, first_entry=0):
        for j in range(first_entry, len(table[b])):
            if table[b][j] >= 0:
                refs[table[b][j]] -= 1
                table[b][j] = -1

    def fork(src, dst):
        drop(dst)
        table[dst] = list(table[src])
        for p in table[src]:
            if p >= 0:
                refs[p] += 1

    def reserve(first, last, keep):
        free, before, granted = [p for p, r in enumerate(refs) if r == 0], list(refs), []
        for b, (lo, hi) in enumerate(zip(first, last)):
            lead = max(hi, 0)
            for j, p in enumerate(list(table[b])):
                wanted = lo < hi and lo // page <= j and j * page < hi
                if wanted and (p < 0 or before[p] > 1):
                    if free:
                        table[b][j] = free.pop(0)
                        refs[table[b][j]] = 1
                        if p >= 0:
                            move(p, table[b][j], max(0, min(page, keep[b] - j * page)))
                            refs[p] -= 1
                    else:
                        lead = min(lead, j * page)
            granted.append(min(lead, len(table[b]) * page))
        return granted

    n, hi = case["seqs"], case["hi"]
    live = None
    if case["op"] == "fork":
        for b in range(1, n):
            fork(0, b)
        granted = reserve([hi] * n, [0] + [hi + 8] * (n - 1), [hi] * n)
    else:
        fork(0, 1)
        granted = reserve([0, 0, 0], [0, hi, 0], [0, hi, 0])
        drop(0)
        holes = [p for p, r in enumerate(refs) if r == 0]
        live = sum(r > 0 for r in refs)
        for p in range(live, len(refs)):
            if refs[p] > 0:
                to = holes.pop(0)
                move(p, to, page)
                refs[to], refs[p] = refs[p], 0
                table = [[to if x == p else x for x in row] for row in table]
        fork(1, 0)
        drop(1)

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")

    out = {"k": k, "v": v, "table": ints(table), "refs": ints(refs), "granted": ints(granted)}
    return out if live is None else dict(out, live=ints([live]))


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "attend":
        return _exact_attend(case, st)
    return _exact_append(case, st) if case["op"] == "append" else _exact_pages(case, st)
