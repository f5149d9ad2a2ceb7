"""Long sums do not drift.  A tensor core's fp32 sum drops what passes its end; were all terms of one sign, a run of hundreds
of pages would come out low by 2^-24 of itself an MMA, which the minima's sum does not.  Keys of nearly equal weights over
16000 tokens, whose mean is a hundredth of a value's spread, show it: fp16 outputs stay within a quarter of their own rounding's
errors (the weights' 22 bits and fp32 sums are a tenth of them), and their mean error within 2^-13 of their size: a run here has
250 pages of 8 MMAs, each off by 2^-24 of a sum that is not larger than the output, on average."""
import pytest
import torch

import paged_ref as R
from paper_2609_26100_gb300 import native, paged

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("b,n,hk,gq,d", [(32, 1, 32, 1, 128), (16, 4, 32, 2, 64), (16, 9, 32, 1, 128), (16, 20, 32, 1, 64), (16, 100, 32, 1, 128),
                                         (16, 16, 32, 4, 128)])
@pytest.mark.parametrize("qscale", [0.0, 1.0])
def test_nearly_equal_weights(b, n, hk, gq, d, qscale):
    first = 16000
    pages = paged.pages_for(first + n)
    g = torch.Generator(device="cuda").manual_seed(n + d)
    c = paged.Kv4Cache.allocate(n_layers=1, n_pages=b * pages, n_seqs=b, max_pages=pages, n_q_heads=hk * gq, n_kv_heads=hk, head_dim=d)
    every = list(range(b))
    c.pages.reserve(every, [first + n] * b)
    for i in every:
        k, v = (torch.randn(first + n, hk, d, generator=g, device="cuda", dtype=torch.float16) for _ in range(2))
        c.append(0, c.batch([i], [0], [first + n]), k, v)
    q = (torch.randn(b * n, hk * gq, d, generator=g, device="cuda") * qscale).half()
    out = torch.empty_like(q)
    c.attention(0, c.batch(every, [first] * b, [n] * b), q, out)
    assert c.sync_status() == native.TSS_OK
    off, size, own = [], [], []
    for seq, head in ((0, 0), (b // 2, hk // 2), (b - 1, hk - 1)):
        k, v = (R.sequence_values(c.pool[0], c.table, seq, first + n, hk, d, side)[:, head] for side in (0, 1))
        for row in range(0, n, max(1, n // 6)):
            for x in range(gq):
                at = seq * n + row
                p = (k[:first + row + 1] @ q[at, head * gq + x].double() * d ** -0.5).softmax(0)
                ref = p @ v[:first + row + 1]
                off.append(out[at, head * gq + x].double() - ref)
                own.append(ref.half().double() - ref)
                size.append(ref)
    off, own, size = (torch.cat(t) for t in (off, own, size))
    rms = lambda t: float(t.square().mean().sqrt())  # noqa: E731
    assert rms(off) <= 1.25 * rms(own), (rms(off), rms(own))
    # (own roundings are of mixed signs: four of their mean's standard deviations)
    assert abs(float(off.mean())) <= 2.0 ** -13 * rms(size) + 4 * rms(own) / len(own) ** 0.5
