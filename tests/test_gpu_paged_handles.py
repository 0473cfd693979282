"""Paged handles where sequences share pages that a round is about to write, and where the pool is short: against
contiguous handles of the same history.

Both hold the same fp32 rows and differ in how attention sums them and in how many rows a projection takes at
once, so logits of equal histories agree to 1e-4 (fp32 weights) and 1e-3 (bf16, as the plane projections'
tests derive)."""
import numpy as np
import pytest
import torch

import sd2_inputs as si
from sd2_inputs.configs import Dims, Workload
from paper_2511_09844_amd import binding as B

pytestmark = pytest.mark.gpu

TOL = {"f32": 1e-4, "bf16": 1e-3}
BF16 = Workload(name="paged-handles", verifier=Dims(1, 768, 12, 4, 1280, 1008, 5e5),
                drafter=Dims(1, 512, 16, 4, 768, 1008, 5e5), dtype="bf16", k=4, batch=4, prompt=(40, 40), new_tokens=30,
                temperature=0.0, seed=5)
F32 = si.TINY.with_(name="paged-handles", batch=4, prompt=(40, 40), new_tokens=30, temperature=0.0, seed=5)


class Model:
    """Weights of a workload on the GPU, for several handles."""

    def __init__(self, wl):
        import gpu_harness
        self.wl = wl
        self.dv, self.dd = gpu_harness.device_model(wl, 0), gpu_harness.device_model(wl, 1)
        self.ws = B.to_device(si.steer_weights(wl))

    def engine(self, paging=None):
        return B.Engine(B.config_of(self.wl), self.dv, self.dd, self.ws, paging=paging)


def prompts(n, length, seed=3):
    return torch.randint(0, 1000, (n, length), generator=torch.Generator().manual_seed(seed), dtype=torch.int32)


def prefill(eng, toks, lens=None):
    lens = [toks.shape[1]] * toks.shape[0] if lens is None else lens
    eng.prefill(toks.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), toks.shape[1])


def close(a, b, tol):
    for name in (B.DBG_LOGITS_V, B.DBG_LOGITS_D, B.DBG_STEER):
        err = np.abs(a.debug(name) - b.debug(name)).max(axis=tuple(range(1, a.debug(name).ndim)))
        assert (err <= tol).all(), (name, err)


def decisions(accepted, k, seed):
    """What a round is forced to: drafts, how many of them are accepted, the token after."""
    g = torch.Generator().manual_seed(seed)
    rows = torch.randint(0, 1000, (len(accepted), k + 2), generator=g, dtype=torch.int32)
    rows[:, k] = torch.tensor(accepted, dtype=torch.int32)
    return rows


def advance(eng, forced):
    out, cnt = eng.round(forced.cuda())
    return out.cpu().tolist(), cnt.cpu().tolist()


@pytest.mark.parametrize("wl", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("length,slot", [(13, 0), (20, 7), (12, 15)], ids=["first", "middle", "last"])
@pytest.mark.parametrize("accepted", [4, 3, 0])
@pytest.mark.parametrize("stream", [False, True], ids=["default", "graphs"])
def test_fork_after_a_round(wl, length, slot, accepted, stream):
    """With every draft accepted the verifier holds one position more than the drafter, on a page that the fork
    shares: that row belongs to what is copied, whatever slot it lies in.  (On a stream of its own rounds are replayed
    from graphs.)"""
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream() if stream else torch.cuda.current_stream()):
        fork_after_a_round(wl, length, slot, accepted)
    torch.cuda.synchronize()


def fork_after_a_round(wl, length, slot, accepted):
    m = Model(wl.with_(prompt=(length, length)))
    plain, paged = m.engine(), m.engine(paging=(16, 40))
    toks = prompts(1, length)
    prefill(plain, toks.expand(4, -1).contiguous())
    prefill(paged, toks)
    first = decisions([accepted], wl.k, 1)
    advance(plain, first.expand(4, -1).contiguous())
    advance(paged, first)
    state = paged.state()[0]
    assert state["len_v"] == length + accepted and state["len_d"] == state["len_v"] - (accepted == wl.k)
    if accepted == wl.k:
        assert state["len_d"] % 16 == slot
    paged.fork(0)
    paged.fork(1, 2)
    for r in range(3):
        forced = decisions([[4, 0, 2, 4], [1, 4, 4, 0], [2, 2, 0, 1]][r], wl.k, 10 + r)
        assert advance(plain, forced) == advance(paged, forced)
        close(plain, paged, TOL[wl.dtype])
        assert plain.state() == paged.state()
        refs, table = paged.debug(B.DBG_REFS), paged.debug(B.DBG_TABLE)
        assert all((table == p).sum() == n for p, n in enumerate(refs))


def generate(eng, n, limit=300):
    """Tokens per sequence until all are done, and how often each sat out a round (which changes nothing of it)."""
    got, waited = [[] for _ in range(n)], [0] * n
    for _ in range(limit):
        before, steer = eng.state(), eng.debug(B.DBG_STEER)
        out, cnt = eng.round()
        out, cnt, after, kept = out.cpu(), cnt.cpu(), eng.state(), eng.debug(B.DBG_STEER)
        for b in range(n):
            if after[b]["done"] == 2:
                waited[b] += 1
                assert int(cnt[b]) == 0 and (out[b] == -1).all() and (kept[b] == steer[b]).all()
                assert {**after[b], "done": 0} == {**before[b], "done": 0}
            got[b] += out[b, : int(cnt[b])].tolist()
        if all(s["done"] == 1 for s in after):
            return got, waited
    raise AssertionError("sequences that cannot go on")


@pytest.mark.parametrize("wl", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("lens", [[17, 18], [18, 17], [17, 18, 18], [18, 17, 18], [17] + 19 * [18], 69 * [18] + [17]], ids=len)
def test_a_sequence_takes_no_pages_of_a_round_it_cannot_run(wl, lens):
    """One free page.  A block of 17 positions that begins a page takes two of 16, any other here one: a sequence that
    needs one goes on, whichever comes first, and the others when it has finished."""
    n = len(lens)
    wl = wl.with_(k=16, new_tokens=10, batch=n, prompt=(17, 18))
    m = Model(wl)
    plain, paged = m.engine(), m.engine(paging=(16, 2 * n))
    toks = prompts(n, 18)
    prefill(plain, toks, lens)
    want, _ = generate(plain, n)
    prefill(paged, toks, lens)
    assert (paged.debug(B.DBG_REFS) == 0).sum() == 1
    got, waited = generate(paged, n)
    assert got == want
    assert waited[lens.index(18)] == 0 and sum(w > 0 for w in waited) == n - 1


@pytest.mark.parametrize("own", [False, True], ids=["drafter", "itself"])
@pytest.mark.parametrize("page,n_pages", [(16, 17), (32, 12)])
@pytest.mark.parametrize("seed", [0, 1, 2])
def test_random_forks_releases_and_compactions(own, page, n_pages, seed):
    """Two prompts and greedy decoding, over a pool that is short at times.  Whatever is forked, released and moved between
    the rounds, each sequence goes on with the tokens of the prompt it comes from.  itself: the verifier drafts, so
    that nearly every draft is accepted."""
    g = torch.Generator().manual_seed(seed)

    def pick(n):
        return int(torch.randint(0, n, (1,), generator=g))

    wl = F32.with_(batch=7, new_tokens=40, prompt=(30, 45))
    if own:
        wl = wl.with_(drafter=wl.verifier)
    m = Model(wl)
    if own:
        m.dd = m.dv
    cfg = B.config_of(wl, steering=B.STEER_NONE) if own else B.config_of(wl)
    ws = None if own else m.ws
    plain, paged = B.Engine(cfg, m.dv, m.dd, ws), B.Engine(cfg, m.dv, m.dd, ws, paging=(page, n_pages))
    toks, lens = prompts(2, 45, seed), [45, 30]
    prefill(plain, toks, lens)
    want, _ = generate(plain, 2)
    prefill(paged, toks, lens)
    origin, got, over, full = [0, 1], [[], []], set(), 0
    for _ in range(200):
        state = paged.state()
        what = pick(6)
        if what == 0 and len(origin) < 7:
            b, count = pick(len(origin)), 1 + pick(min(2, 7 - len(origin)))
            paged.fork(b, count)
            origin += [origin[b]] * count
            got += [list(got[b]) for _ in range(count)]
            if state[b]["done"] == 1:
                over |= set(range(len(origin) - count, len(origin)))
        elif what == 1:
            paged.compact()
        elif what == 2 and len(origin) > 3:
            b = 2 + pick(len(origin) - 2)
            paged.release(b)
            over.add(b)
        before = paged.state()
        out, cnt = (x.cpu().tolist() for x in paged.round())
        after = paged.state()
        for b in range(len(origin)):
            got[b] += out[b][: cnt[b]]
            full += cnt[b] == wl.k + 1
            assert got[b] == want[origin[b]][: len(got[b])], b
            if after[b]["done"] == 1 and b not in over:
                assert got[b] == want[origin[b]]
                over.add(b)
            if before[b]["done"] == 1:
                assert cnt[b] == 0
        refs, table = paged.debug(B.DBG_REFS), paged.debug(B.DBG_TABLE)
        assert all((table == p).sum() == n for p, n in enumerate(refs))
        if len(over) == len(origin):
            break
        if all(s["done"] for s in after):
            b = max(b for b in range(len(origin)) if b not in over)
            paged.release(b)
            over.add(b)
    assert len(over) == len(origin)
    assert not own or full > 8
