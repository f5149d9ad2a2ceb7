"""The stage of the ring through which a warp's part of an item is joined takes a page's copy right after: runs of many
short items, each with a value of its own, return it in every call, for one and for two tiles of rows."""
import pytest
import torch

from paper_2609_26100_gb300 import native, paged

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,d", [(1, 128), (1, 64), (8, 128), (9, 128), (16, 64)])
@pytest.mark.parametrize("first", [0, 31, 120, 250])
def test_short_items_in_long_runs(rows, d, first):
    b, h = 64, 48
    tokens = first + rows
    pages = paged.pages_for(tokens)
    c = paged.Kv4Cache.allocate(n_layers=1, n_pages=b * pages, n_seqs=b, max_pages=pages, n_q_heads=h, n_kv_heads=h, head_dim=d)
    every = list(range(b))
    c.pages.reserve(every, [tokens] * b)
    g = torch.Generator(device="cuda").manual_seed(rows + first)
    # all tokens of a (sequence, head) hold one value: a scale of 0 and that minimum
    one = torch.randint(-2000, 2000, (b, 1, h, 1), generator=g, device="cuda").float()
    k = torch.randn(b * tokens, h, d, generator=g, device="cuda", dtype=torch.float16)
    v = one.expand(b, tokens, h, d).reshape(b * tokens, h, d).half()
    c.append(0, c.batch(every, [0] * b, [tokens] * b), k, v)
    q = torch.randn(b * rows, h, d, generator=g, device="cuda", dtype=torch.float16)
    batch = c.batch(every, [first] * b, [rows] * b)
    want = one.expand(b, rows, h, d).reshape(b * rows, h, d)
    out = torch.empty_like(q)
    for _ in range(25):
        c.attention(0, batch, q, out.fill_(0.5))
        # sum p z / sum p of equal z: 2^-22 or so, then half an ulp of fp16 (integers below 2048 are exact in it)
        assert ((out.float() - want).abs() <= want.abs() * 2.0 ** -11).all()
    assert c.sync_status() == native.TSS_OK
