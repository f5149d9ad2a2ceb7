"""Windows, first tokens and positions at the ends of 32 bits."""
import pytest
import torch

from paper_2609_26100_gb300 import native, paged

pytestmark = pytest.mark.gpu
MOST = 2 ** 31 - 1


@pytest.mark.parametrize("d,n", [(128, 5), (128, 90), (64, 90)])
@pytest.mark.parametrize("positions", [False, True])
def test_a_window_of_everything(d, n, positions):
    """A window (or first tokens) as large as an int holds what no window holds, for masks that name later rows too."""
    h, first = 2, 150
    c = paged.Kv4Cache.allocate(n_layers=1, n_pages=8, n_seqs=1, max_pages=8, n_q_heads=h, n_kv_heads=h, head_dim=d)
    c.pages.reserve([0], [first + n])
    g = torch.Generator(device="cuda").manual_seed(d + n)
    kv = torch.randn(first + n, h, d, generator=g, device="cuda", dtype=torch.float16)
    c.append(0, c.batch([0], [0], [first + n]), kv, kv.flip(0))
    q = torch.randn(n, h, d, generator=g, device="cuda", dtype=torch.float16)
    mask = torch.full((n, 2), -1, dtype=torch.int64, device="cuda")  # every row sees the whole block
    b = c.batch([0], [first], [n])
    want, got = torch.empty_like(q), torch.empty_like(q)
    c.attention(0, b, q, want, mask=mask)
    pos = torch.full((n,), first, dtype=torch.int32, device="cuda") if positions else None
    for window, sinks in ((MOST, 0), (MOST, MOST), (1, MOST)):
        c.attention(0, b, q, got.fill_(3.0), mask=mask, window=window, sinks=sinks, positions=pos)
        assert torch.equal(got, want), (window, sinks)
    assert c.sync_status() == native.TSS_OK


@pytest.mark.parametrize("n", [3, 60])
def test_positions_far_past_the_context(n):
    """A row whose position is the largest int sees, under a window, nothing but itself (at the same position)."""
    h, d, first = 2, 128, 130
    c = paged.Kv4Cache.allocate(n_layers=1, n_pages=8, n_seqs=1, max_pages=8, n_q_heads=h, n_kv_heads=h, head_dim=d)
    c.pages.reserve([0], [first + n])
    g = torch.Generator(device="cuda").manual_seed(n)
    kv = torch.randn(first + n, h, d, generator=g, device="cuda", dtype=torch.float16)
    c.append(0, c.batch([0], [0], [first + n]), kv, kv)
    held = torch.empty(first + n, h, d, device="cuda")
    c.read(0, c.batch([0], [0], [first + n]), None, held)
    q = torch.randn(n, h, d, generator=g, device="cuda", dtype=torch.float16)
    pos = torch.arange(MOST - n + 1, MOST + 1, device="cuda").to(torch.int32)
    out = torch.empty_like(q)
    c.attention(0, c.batch([0], [first], [n]), q, out, window=1, positions=pos)
    # one key: its value, rounded to fp16 after weights of 22 bits
    err = (out.float() - held[first:]).abs()
    assert (err <= held[first:].abs() * 2.0 ** -11 + 2.0 ** -14).all()
    assert c.sync_status() == native.TSS_OK
