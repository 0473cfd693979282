"""What PagedCache refuses beside sizes and types: gradients that would be lost, and operands that lie in one another."""
import pytest
import torch
import torch.autograd.forward_ad as forward_ad

from paged_ref import attend64, attend_bound, make_cache

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def setup():
    cache = make_cache([40, 50], BF16, 2, 64, 16)
    ln = torch.tensor([40, 50], dtype=torch.int32, device="cuda")
    q = torch.randn(2, 4, 64, generator=torch.Generator().manual_seed(1)).to(BF16).cuda()
    return cache, ln, q


def refused(call):
    from paper_2511_09844_amd.binding import Sd2Error
    with pytest.raises(Sd2Error):
        call()


def test_forward_mode_tangents_are_refused():
    cache, ln, q = setup()
    kv = q[:, :2].contiguous()
    with forward_ad.dual_level():
        dual, rows = forward_ad.make_dual(q, torch.ones_like(q)), forward_ad.make_dual(kv, torch.ones_like(kv))
        refused(lambda: cache.attend(dual, ln))
        refused(lambda: cache.append(rows, kv, ln))
        refused(lambda: cache.append(kv, rows, ln))
        with torch.no_grad():  # (which does not stop forward mode)
            refused(lambda: cache.attend(dual, ln))
        plain = cache.attend(q, ln)  # no tangent, no refusal
    assert torch.equal(plain, cache.attend(forward_ad.unpack_dual(dual).primal, ln))


def test_pools_that_want_gradients_are_refused():
    from paper_2511_09844_amd.paged import PagedCache
    cache, ln, q = setup()
    for k, v in ((cache.k.clone().requires_grad_(), cache.v), (cache.k, cache.v.clone().requires_grad_())):
        refused(lambda: PagedCache(k, v, cache.table, cache.refs))
        with torch.no_grad():
            refused(lambda: PagedCache(k, v, cache.table, cache.refs))  # (it may be used outside)
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(cache.k, torch.ones_like(cache.k))
        refused(lambda: PagedCache(dual, cache.v, cache.table, cache.refs))
    assert torch.equal(PagedCache(cache.k, cache.v, cache.table, cache.refs).attend(q, ln), cache.attend(q, ln))


@pytest.mark.parametrize("rows", [1, 70])
def test_q_and_out_that_share_elements_are_refused(rows):
    """Columns of one buffer: heads 0-3 are q; out beside them is computed, out over them refused."""
    cache = make_cache([rows + 40, rows + 9], BF16, 2, 64, 16)
    ln = torch.tensor([rows + 40, rows + 9], dtype=torch.int32, device="cuda")
    wide = torch.randn(2 * rows, 12, 64, generator=torch.Generator().manual_seed(1)).to(BF16).cuda()
    q = wide[:, 4:8]
    want = cache.attend(q, ln)
    ref, absv, spread = attend64(cache, q, [rows + 40, rows + 9], [rows] * 2)
    assert ((want.double() - ref).abs() <= attend_bound(ref, absv, spread, BF16, rows + 40, 64)).all()
    for first in (1, 2, 3, 4, 5, 7):
        refused(lambda: cache.attend(q, ln, out=wide[:, first: first + 4]))
    for first in (0, 8):
        assert torch.equal(cache.attend(q, ln, out=wide[:, first: first + 4]), want)
    assert torch.equal(cache.attend(q, ln), want)
    flat = torch.empty(4 * rows, 4, 64, dtype=BF16, device="cuda")  # one behind the other
    flat[: 2 * rows] = q
    assert torch.equal(cache.attend(flat[: 2 * rows], ln, out=flat[2 * rows:]), want)
    refused(lambda: cache.attend(flat[: 2 * rows], ln, out=flat[2 * rows - 1: 4 * rows - 1]))
