"""Handles whose caches lie in pages: rounds against the CPU oracle, and forks, releases, compaction and a
pool that runs out against handles that have the room.

The paged and the contiguous caches hold the same fp32 rows and differ in how attention sums them, so
logits of equal histories agree to the oracle tests' tolerances."""
import functools

import numpy as np
import pytest
import torch

import sd2_inputs as si
from sd2_inputs.configs import Dims, Workload
from paper_2511_09844_amd import binding as B

pytestmark = pytest.mark.gpu

VER = Dims(1, 768, 12, 4, 1280, 1008, 5e5)
DRF = Dims(1, 512, 16, 4, 768, 1008, 5e5)


def parity(monkeypatch, wl, page, n_pages, **kw):
    import gpu_harness
    monkeypatch.setattr(gpu_harness.B, "Engine", functools.partial(B.Engine, paging=(page, n_pages)))
    st = gpu_harness.parity_run(wl, expect_path=0, **kw)
    assert st.pinned > 0
    return st


def pool(wl, page):
    """Pages that every sequence of a workload needs at its end."""
    return wl.batch * -(-wl.max_seq_len // page)


@pytest.mark.parametrize("page", [16, 64])
def test_tiny_f32(monkeypatch, page):
    parity(monkeypatch, si.TINY, page, pool(si.TINY, page))


@pytest.mark.parametrize("unsteered", [False, True])
def test_f32_ragged_batch(monkeypatch, unsteered):
    wl = si.TINY.with_(name="paged-f32", batch=5, prompt=(1, 70), new_tokens=12, seed=11)
    parity(monkeypatch, wl, 32, pool(wl, 32), unsteered=unsteered)


@pytest.mark.parametrize("batch,k,prompt,page", [(1, 4, (129, 129), 16), (3, 10, (1, 90), 32), (7, 5, (200, 300), 64),
                                                 (16, 7, (1, 40), 128), (2, 16, (17, 900), 256)])
def test_bf16_batches(monkeypatch, batch, k, prompt, page):
    wl = Workload(name="paged", verifier=VER, drafter=DRF, dtype="bf16", temperature=1.0, batch=batch, k=k, prompt=prompt,
                  new_tokens=k + 3, seed=31 + batch)
    st = parity(monkeypatch, wl, page, pool(wl, page), seqs=sorted({0, batch // 2, batch - 1}))
    assert max(st.max_err_v, st.max_err_d, st.max_err_s) <= 1e-3  # as the plane projections' tests derive


def test_bf16_prefill_in_chunks(monkeypatch):
    # 2048 rows a chunk over ragged prompts, several chunks
    wl = Workload(name="paged-chunks", verifier=Dims(1, 1024, 8, 8, 2048, 1008, 5e5),
                  drafter=Dims(1, 512, 8, 8, 1024, 1008, 5e5), dtype="bf16", temperature=1.0, batch=5, k=3, prompt=(1, 900),
                  new_tokens=5, seed=101)
    parity(monkeypatch, wl, 64, pool(wl, 64), seqs=[0, 2, 4])


# ---- forks, releases, compaction, a small pool -----------------------------------------------------------

class Model:
    """Weights of a workload on the GPU, for several handles."""

    def __init__(self, wl):
        import gpu_harness
        self.wl = wl
        self.dv, self.dd = gpu_harness.device_model(wl, 0), gpu_harness.device_model(wl, 1)
        self.ws = B.to_device(si.steer_weights(wl))

    def engine(self, paging=None, **cfg):
        return B.Engine(B.config_of(self.wl, **cfg), self.dv, self.dd, self.ws, paging=paging)


def prompts(n, length, seed=3):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(0, 1000, (n, length), generator=g, dtype=torch.int32)


def prefill(eng, toks, lens=None):
    lens = [toks.shape[1]] * toks.shape[0] if lens is None else lens
    eng.prefill(toks.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), toks.shape[1])


def close(a, b, what, tol=1e-4):
    for name in (B.DBG_LOGITS_V, B.DBG_LOGITS_D, B.DBG_STEER):
        err = np.abs(a.debug(name)[what] - b.debug(name)[what]).max()
        assert err <= tol, (name, err)


WL = si.TINY.with_(name="paged-calls", batch=4, prompt=(40, 40), new_tokens=30, seed=5)


def test_forked_sequences_are_the_same_prompt_several_times():
    m = Model(WL)
    one, four = m.engine(paging=(16, 40)), m.engine()
    toks = prompts(1, 40)
    prefill(one, toks)
    one.fork(0)
    one.fork(1, 2)
    assert one.batch == 4
    prefill(four, toks.expand(4, -1).contiguous())
    refs = one.debug(B.DBG_REFS)
    assert sorted(refs[refs > 0].tolist()) == [4, 4, 4]  # 39 cached positions in three shared pages
    for _ in range(4):
        out, cnt = four.round()
        forced = np.concatenate([four.debug(B.DBG_OWN_DRAFTS), four.debug(B.DBG_OWN_N)[:, None], four.debug(B.DBG_OWN_Y)[:, None]], 1)
        out1, cnt1 = one.round(torch.from_numpy(forced.astype(np.int32)).cuda())
        assert torch.equal(out, out1) and torch.equal(cnt, cnt1)
        close(one, four, slice(None))
        assert one.state() == four.state()
    draws = four.debug(B.DBG_OWN_DRAFTS)
    assert (draws != draws[:1]).any()  # random numbers of their own
    refs, table = one.debug(B.DBG_REFS), one.debug(B.DBG_TABLE)
    for p, r in enumerate(refs):
        assert (table == p).sum() == r
    # the two full pages of the prompt are still shared, the third was written to
    assert sorted(refs[refs > 1].tolist()) == [4, 4]


def generate(eng, n, rounds=None, between=None):
    """Emitted tokens per sequence."""
    got = [[] for _ in range(n)]
    r = 0
    while not all(s["done"] == 1 for s in eng.state()) and (rounds is None or r < rounds):
        out, cnt = eng.round()
        out, cnt = out.cpu(), cnt.cpu()
        for b in range(len(cnt)):
            got[b] += out[b, : int(cnt[b])].tolist()
        r += 1
        assert r < 200
        if between:
            between(r)
    return got


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_greedy_generation_with_compaction_and_a_fork_on_the_way(dtype):
    wl = WL.with_(temperature=0.0) if dtype == "f32" else Workload(
        name="paged-greedy", verifier=VER, drafter=DRF, dtype="bf16", k=4, batch=4, prompt=(40, 40), new_tokens=30,
        temperature=0.0, seed=5)
    m = Model(wl)
    plain, paged = m.engine(), m.engine(paging=(16, 24))
    toks, lens = prompts(3, 40), [40, 23, 31]
    prefill(plain, toks, lens)
    want = generate(plain, 3)
    prefill(paged, toks, lens)
    seen = {}

    def between(r):
        if r == 2:
            seen["t"] = paged.state()[1]["t"]
            paged.fork(1)
        if r in (1, 3, 4):
            before = paged.debug(B.DBG_REFS)
            live = int(paged.compact().item())
            after = paged.debug(B.DBG_REFS)
            assert live == (before > 0).sum() and (after[:live] > 0).all() and (after[live:] == 0).all()

    got = generate(paged, 4, between=between)
    assert got[:3] == want
    # the fork goes on as the sequence it came from: greedy, so with the same tokens
    assert got[3] == want[1][seen["t"] - 23:]
    paged.round()  # (finished sequences have given up their pages by the next round)
    assert (paged.debug(B.DBG_REFS) == 0).all()
    # the handle starts again
    prefill(paged, toks, lens)
    assert generate(paged, 3) == want


@pytest.mark.parametrize("n_pages", [8, 9])
def test_a_pool_that_runs_out(n_pages):
    """Two prompts of three pages that grow to five.  Nine pages: the second sequence waits for the first to
    finish.  Eight: at four pages each neither can go on until the caller releases one."""
    m = Model(WL.with_(temperature=0.0))
    plain, paged = m.engine(), m.engine(paging=(16, n_pages))
    toks = prompts(2, 40)
    prefill(plain, toks)
    want = generate(plain, 2)
    prefill(paged, toks)
    stalled, got = 0, [[], []]
    for _ in range(60):
        before = paged.state()
        out, cnt = paged.round()
        after = paged.state()
        for b in range(2):
            if after[b]["done"] == 2:
                stalled += 1
                assert int(cnt[b]) == 0 and {**after[b], "done": 0} == {**before[b], "done": 0}
            got[b] += out[b, : int(cnt[b])].tolist()
        if all(s["done"] == 1 for s in after):
            break
        if all(s["done"] == 2 for s in after):
            assert n_pages == 8
            paged.release(0)
            want[0] = want[0][: len(got[0])]
    assert stalled > 0 and got == want and all(s["done"] == 1 for s in paged.state())


def test_release_makes_room():
    m = Model(WL.with_(temperature=0.0))
    plain, paged = m.engine(), m.engine(paging=(16, 8))
    toks = prompts(2, 40)
    prefill(plain, toks)
    want = generate(plain, 2)
    prefill(paged, toks)
    paged.fork(0)  # a third sequence that shares the first one's pages
    first = generate(paged, 3, rounds=1)
    paged.release(0)
    paged.release(2)
    assert [s["done"] for s in paged.state()] == [1, paged.state()[1]["done"], 1]
    table = paged.debug(B.DBG_TABLE)
    assert (table[0] == -1).all() and (table[2] == -1).all()
    rest = generate(paged, 3)
    assert first[1] + rest[1] == want[1] and rest[0] == [] and rest[2] == []


def test_calls_refused():
    m = Model(WL)
    plain, paged = m.engine(), m.engine(paging=(16, 8))
    lib = plain.lib
    toks = prompts(4, 40)
    assert lib.sd2_fork(paged.h, 0, 1) == -3 and lib.sd2_release(paged.h, 0) == -3 and lib.sd2_compact(paged.h, None) == -3
    with pytest.raises(B.Sd2Error):
        prefill(paged, toks)  # 4 prompts of three pages
    prefill(plain, toks)
    assert lib.sd2_fork(plain.h, 0, 1) == -5 and lib.sd2_release(plain.h, 0) == -5 and lib.sd2_compact(plain.h, None) == -5
    prefill(paged, toks[:2])
    assert lib.sd2_fork(paged.h, 2, 1) == -1 and lib.sd2_fork(paged.h, -1, 1) == -1 and lib.sd2_fork(paged.h, 0, 0) == -1
    assert lib.sd2_fork(paged.h, 0, 3) == -2 and lib.sd2_release(paged.h, 2) == -1
    with pytest.raises(B.Sd2Error):
        paged.train_loss(toks[0].cuda(), torch.ones(40, dtype=torch.int32).cuda(), 16)
    with pytest.raises(B.Sd2Error):
        plain.debug(B.DBG_REFS)


def test_rounds_replayed_from_a_graph():
    """On a stream of its own a round is recorded once and replayed; pages and lengths change under it."""
    m = Model(WL.with_(temperature=0.0))
    plain = m.engine()
    toks = prompts(3, 40)
    prefill(plain, toks)
    want = generate(plain, 3)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        paged = B.Engine(B.config_of(m.wl), m.dv, m.dd, m.ws, stream=s, paging=(16, 24))
        prefill(paged, toks)

        def between(r):
            if r % 2:
                paged.compact()

        assert generate(paged, 3, between=between) == want
    torch.cuda.synchronize()
