"""A wait that runs out in a CTA whose run goes on with other items: the call ends after one bounded wait, says so, and the
next calls are right."""
import time

import pytest
import torch

from paper_2609_26100_gb300 import native, paged

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("b,rows,h,d,first", [(64, 1, 40, 128, 20), (64, 1, 40, 64, 20), (32, 3, 80, 128, 130), (40, 12, 40, 128, 70),
                                              (30, 20, 30, 64, 40), (40, 60, 16, 128, 150)])
def test_short_items(b, rows, h, d, first):
    pages = paged.pages_for(first + rows)
    c = paged.Kv4Cache.allocate(n_layers=1, n_pages=b * pages, n_seqs=b, max_pages=pages, n_q_heads=h, n_kv_heads=h, head_dim=d)
    every = list(range(b))
    c.pages.reserve(every, [first + rows] * b)
    g = torch.Generator(device="cuda").manual_seed(rows)
    kv = torch.randn(b * (first + rows), h, d, generator=g, device="cuda", dtype=torch.bfloat16)
    c.append(0, c.batch(every, [0] * b, [first + rows] * b), kv, kv)
    q = torch.randn(b * rows, h, d, generator=g, device="cuda", dtype=torch.bfloat16)
    batch = c.batch(every, [first] * b, [rows] * b)
    want, want_lse = torch.empty_like(q), torch.empty(b * rows, h, device="cuda")
    c.attention(0, batch, q, want, lse=want_lse)
    assert c.sync_status() == native.TSS_OK and not want.isnan().any()
    for _ in range(2):
        out, lse = torch.empty_like(want), torch.empty_like(want_lse)
        c.inject_timeout(1)
        began = time.perf_counter()
        c.attention(0, batch, q, out, lse=lse)
        assert c.sync_status() == native.TSS_ERR_TIMEOUT
        assert time.perf_counter() - began < 3.5  # (one wait of 2 s, not one an item)
        for _ in range(2):
            c.attention(0, batch, q, out.fill_(9.0), lse=lse.fill_(9.0))
            assert c.sync_status() == native.TSS_OK
            assert torch.equal(out, want) and torch.equal(lse, want_lse)
