"""Freeing with counts past every sequence's pages, up to the largest int, gives nothing back and touches nothing."""
import pytest
import torch

from paper_2609_26100_gb300 import native, paged

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("max_pages", [3, 700])
@pytest.mark.parametrize("keep", [2 ** 31 - 1, 2 ** 31 - 2, 2 ** 31 - 255, 2 ** 30])
def test_counts_past_the_pages(max_pages, keep):
    n = 5
    pool = torch.zeros(1, n * max_pages, 16, dtype=torch.uint8, device="cuda")
    table = torch.full((n, max_pages), -1, dtype=torch.int32, device="cuda")
    p = paged.PagePool(pool, table, torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n * max_pages, dtype=torch.int32, device="cuda"))
    p.reserve([0, 2, 4], [64 * max_pages, 64, 0])
    want = [t.clone() for t in (p.table, p.held, p.refs)]
    p.free([4, 0, 2], [64 * keep] * 3)
    assert p.sync_status() == native.TSS_OK
    assert all(torch.equal(a, b) for a, b in zip(want, (p.table, p.held, p.refs)))
    p.free([0, 2], [64 * keep, 0])  # (beside one that does give pages back)
    assert p.sync_status() == native.TSS_OK
    assert p.held.tolist() == [max_pages, 0, 0, 0, 0] and int(p.refs.sum()) == max_pages
