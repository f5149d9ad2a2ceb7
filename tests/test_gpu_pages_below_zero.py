"""Lengths below zero are refused before anything is launched, those too that round up to no page."""
import pytest

from paper_2609_26100_gb300 import native, paged

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens", [-1, -63, -64, -10 ** 6])
def test_lengths_below_zero(tokens):
    c = paged.Kv4Cache.allocate(n_layers=1, n_pages=6, n_seqs=3, max_pages=2, n_q_heads=1, n_kv_heads=1, head_dim=64)
    c.pages.reserve([0, 1], [100, 20])
    for call in (lambda: c.pages.free([0, 1], [tokens, 20]), lambda: c.pages.reserve([0, 2], [100, tokens]),
                 lambda: c.pages.fork([0], [2], [tokens])):
        with pytest.raises(native.TssError) as e:
            call()
        assert e.value.status == native.TSS_ERR_INVALID_ARG
    assert c.pages.held.tolist() == [2, 1, 0] and c.pages.sync_status() == native.TSS_OK
