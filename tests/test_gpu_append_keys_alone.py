"""The joined append of keys alone (no query heads), where its warps do not fill the last CTA: two warps a half page and KV head, four a
CTA.  A spare warp has no row: pages and keys get the bits of the two separate calls, and nothing is recorded, whatever lies before the
positions."""
import pytest
import torch

from paper_2609_26100_gb300 import native
from test_gpu_append_rope import rows_of, table_of
from test_gpu_paged import make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("d,rot,inter", [(128, 128, False), (128, 128, True), (128, 64, False), (64, 64, False)])
@pytest.mark.parametrize("hk,first,n", [(1, (0,), (1,)), (3, (40,), (1,)), (1, (31,), (40,)), (1, (5, 64, 97), (1, 2, 1)), (3, (0, 1, 2), (1, 1, 1)), (5, (63,), (1,))])
@pytest.mark.parametrize("keep_k", [False, True])
def test_spare_warps(dtype, d, rot, inter, hk, first, n, keep_k):
    lens, rows = [f + m for f, m in zip(first, n)], sum(n)
    assert sum(-(-(f + m) // 32) - f // 32 for f, m in zip(first, n) if m) * 2 * hk % 4  # (else no warp is spare)
    one, two = (make(lens, hk, hk, d) for _ in range(2))
    _, k, v = rows_of(rows, 0, hk, d, dtype, 4)
    t = table_of(rot, 200)
    store = torch.full((64 + rows,), 1 << 30, dtype=torch.int32, device="cuda")  # (positions that no table has, before those meant)
    pos = store[64:]
    pos[:] = torch.cat([torch.arange(f, f + m, device="cuda") for f, m in zip(first, n)])
    ko, ko2 = (torch.empty(k.shape, dtype=dtype, device="cuda") for _ in range(2))
    kw = dict(interleaved=inter)
    one.append_rope(0, one.batch(list(range(len(n))), first, n), native.rope_args(None, k, None, ko if keep_k else None, pos, t, to_pages=True, **kw), v)
    native.qk_rope(native.rope_args(None, k, None, ko2, pos, t, **kw))
    two.append(0, two.batch(list(range(len(n))), first, n), ko2, v)
    assert one.sync_status() == native.TSS_OK and two.sync_status() == native.TSS_OK
    assert torch.equal(one.pool, two.pool)
    if keep_k:
        assert torch.equal(ko, ko2)
