"""The paged attention's bounded waits run out without a GPU fault, the status says so, and the next call is right."""
import pytest
import torch

import paged_ref as R
from paper_2609_26100_gb300 import native
from test_gpu_paged import close, fill, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,hq", [(1, 2), (12, 2), (61, 4)])
def test_a_wait_runs_out_and_the_next_call_is_right(rows, hq):
    first = 700
    cache = make([first + rows], hq, 2, 128)
    k, v = fill(cache, [first + rows])
    q = torch.randn(rows, hq, 128, device="cuda", dtype=torch.bfloat16)
    out, lse = torch.empty_like(q), torch.empty(rows, hq, device="cuda")
    batch = cache.batch([0], [first], [rows])
    cache.inject_timeout(1)
    cache.attention(0, batch, q, out, lse=lse)
    assert cache.sync_status() == native.TSS_ERR_TIMEOUT
    for _ in range(2):
        cache.attention(0, batch, q, out, lse=lse)
        assert cache.sync_status() == native.TSS_OK
        see = R.sees(first, rows, None, range(first, first + rows), 0, 0, "cuda")
        ref, ref_lse = R.attention(k[0], v[0], q.double(), see, 128 ** -0.5)
        close(out, lse, ref, ref_lse, float(v[0].abs().amax()), 40.0)


def test_refusals():
    cache = make([64], 2, 2, 64)
    with pytest.raises(native.TssError):
        cache.inject_timeout(-1)
    cache.inject_timeout(3)
    cache.inject_timeout(0)
    q = torch.randn(1, 2, 64, device="cuda", dtype=torch.bfloat16)
    fill(cache, [64])
    cache.attention(0, cache.batch([0], [63], [1]), q, q.clone())
    assert cache.sync_status() == native.TSS_OK
