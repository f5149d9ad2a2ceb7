"""Windows shorter than a page for rows whose positions end at the largest int: the context's pages that stand
before the window are hidden from every row, whatever page or half page the window's first key of the block falls in."""
import pytest
import torch

import paged_ref as R
from paper_2609_26100_gb300 import native, paged

pytestmark = pytest.mark.gpu
MOST = 2 ** 31 - 1


@pytest.mark.parametrize("d,n", [(128, 3), (128, 20), (128, 60), (64, 3), (64, 60)])
@pytest.mark.parametrize("window", [10, 31, 40, 63, 64, 100])
@pytest.mark.parametrize("first", [66, 128, 130, 170])
def test_a_row_at_the_largest_position(d, n, window, first):
    h = 2
    c = paged.Kv4Cache.allocate(n_layers=1, n_pages=8, n_seqs=1, max_pages=8, n_q_heads=h, n_kv_heads=h, head_dim=d)
    c.pages.reserve([0], [first + n])
    g = torch.Generator(device="cuda").manual_seed(n + window)
    k, v = (torch.randn(first + n, h, d, generator=g, device="cuda", dtype=torch.float16) for _ in range(2))
    c.append(0, c.batch([0], [0], [first + n]), k, v)
    k, v = (R.sequence_values(c.pool[0], c.table, 0, first + n, h, d, side) for side in (0, 1))
    q = torch.randn(n, h, d, generator=g, device="cuda", dtype=torch.float16)
    pos = list(range(MOST - n + 1, MOST + 1))
    out, lse = torch.empty_like(q), torch.empty(n, h, device="cuda")
    c.attention(0, c.batch([0], [first], [n]), q, out, lse=lse, window=window, positions=torch.tensor(pos, dtype=torch.int32, device="cuda"))
    assert c.sync_status() == native.TSS_OK
    ref, ref_lse = R.attention(k, v, q.double(), R.sees(first, n, None, pos, window, 0, "cuda"), d ** -0.5)
    # (fp16 outputs: half an ulp, and weights of 11 bits or more; scores of a few units in fp32)
    assert ((out.double() - ref).abs() <= ref.abs() * 2.0 ** -11 + float(v.abs().amax()) * 2.0 ** -10).all()
    assert ((lse.double() - ref_lse).abs() <= 2e-4).all()


def test_whole_pages_as_units():
    """As many requests and heads as give every warp several pages: a row alone sees itself, whose value it returns."""
    b, h, d, first = 64, 40, 64, 150
    c = paged.Kv4Cache.allocate(n_layers=1, n_pages=3 * b, n_seqs=b, max_pages=3, n_q_heads=h, n_kv_heads=h, head_dim=d)
    c.pages.reserve(list(range(b)), [first + 1] * b)
    g = torch.Generator(device="cuda").manual_seed(1)
    kv = torch.randn(b * (first + 1), h, d, generator=g, device="cuda", dtype=torch.float16)
    c.append(0, c.batch(list(range(b)), [0] * b, [first + 1] * b), kv, kv)
    own = torch.empty(b, h, d, device="cuda")
    batch = c.batch(list(range(b)), [first] * b, [1] * b)
    c.read(0, batch, None, own)
    q = torch.randn(b, h, d, generator=g, device="cuda", dtype=torch.float16)
    pos, out = torch.full((b,), MOST, dtype=torch.int32, device="cuda"), torch.empty_like(q)
    for window in (30, 63, 64):
        c.attention(0, batch, q, out.fill_(9.0), window=window, positions=pos)
        # one key: its value, rounded to fp16 after weights of 22 bits
        assert ((out.float() - own).abs() <= own.abs() * 2.0 ** -11 + 2.0 ** -14).all(), window
    assert c.sync_status() == native.TSS_OK
