"""Paged calls at the ends of the documented sizes."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_more_entries_asked_for_than_32_bits_count():
    """48 sequences ask for 45 million entries each, 2^31 and more in all, of a pool of seven pages."""
    from paper_2511_09844_amd.paged import PagedCache
    seqs, entries, n_pages = 48, 45_000_000, 7
    assert seqs * entries > 2 ** 31
    cache = PagedCache.empty(n_pages, 16, 1, 1, 32, seqs, entries)
    last = torch.full((seqs,), 16 * entries, dtype=torch.int32, device="cuda")
    granted = cache.reserve(torch.zeros_like(last), last)
    assert granted.tolist() == [16 * n_pages] + [0] * (seqs - 1)
    assert cache.refs.tolist() == [1] * n_pages
    assert cache.table[0, :n_pages].tolist() == list(range(n_pages))
    assert sum(int((row >= 0).sum()) for row in cache.table) == n_pages
