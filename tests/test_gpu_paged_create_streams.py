"""Workspaces made while the default stream has work in front are ready for calls on another stream at once."""
import pytest
import torch

from paper_2609_26100_gb300 import native, paged

pytestmark = pytest.mark.gpu


def test_created_behind_a_busy_default_stream():
    h, d, first = 4, 128, 3000
    pages = paged.pages_for(first + 1)
    pool = torch.zeros(1, pages, paged.page_bytes(h, d), dtype=torch.uint8, device="cuda")
    table = torch.full((1, pages), -1, dtype=torch.int32, device="cuda")
    held, refs = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(pages, dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    kv = torch.randn(first + 1, h, d, generator=g, device="cuda", dtype=torch.bfloat16)
    q = torch.randn(1, h, d, generator=g, device="cuda", dtype=torch.bfloat16)
    outs = [torch.empty_like(q) for _ in range(2)]

    def use(out):
        c = paged.Kv4Cache(pool, table, n_q_heads=h, n_kv_heads=h, head_dim=d)
        c.pages = paged.PagePool(pool, table, held, refs)
        c.pages.free([0])
        c.pages.reserve([0], [first + 1])
        c.append(0, c.batch([0], [0], [first + 1]), kv, kv)
        c.attention(0, c.batch([0], [first], [1]), q, out)
        assert c.sync_status() == native.TSS_OK and c.pages.sync_status() == native.TSS_OK
        return c

    use(outs[0]).close()
    side = torch.cuda.Stream()
    for _ in range(5):
        # memory that workspaces are likely to get is full of ones, and what would clear them there stands in a queue
        junk = torch.full((1 << 24,), -1, dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        del junk
        torch.cuda.empty_cache()
        torch.cuda._sleep(100_000_000)  # (some 50 ms)
        with torch.cuda.stream(side):
            c = use(outs[1].fill_(9.0))
            side.synchronize()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1])
        assert c.sync_status() == native.TSS_OK and c.pages.sync_status() == native.TSS_OK
        c.close()
