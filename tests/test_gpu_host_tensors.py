"""Tensors in host memory are refused before anything is launched, and the rotary table is filled on torch's
current stream."""
import pytest
import torch

from paper_2609_26100_gb300 import native, paged

pytestmark = pytest.mark.gpu
H, D = 2, 64


def _cache():
    return paged.Kv4Cache.allocate(n_layers=1, n_pages=4, n_seqs=1, max_pages=2, n_q_heads=H, n_kv_heads=H, head_dim=D)


def test_cache_calls():
    c = _cache()
    b = c.batch([0], [0], [3])
    here = torch.ones(3, H, D, dtype=torch.bfloat16)
    there = here.cuda()
    c.pages.reserve([0], [3])
    for k, v in ((here, there), (there, here)):
        with pytest.raises(ValueError):
            c.append(0, b, k, v)
        with pytest.raises(ValueError):
            c.read(0, b, k, v)
    c.append(0, b, there, there)
    out = torch.empty_like(there)
    for q, o, extra in ((here, here, {}), (there, out, {"lse": torch.empty(3, H)}), (there, out, {"mask": torch.zeros(3, 2, dtype=torch.int64)}),
                        (there, out, {"window": 4, "positions": torch.zeros(3, dtype=torch.int32)})):
        with pytest.raises(ValueError):
            c.attention(0, b, q, o, **extra)
    assert c.sync_status() == native.TSS_OK


def test_pools_and_tables():
    c = _cache()
    ints = dict(dtype=torch.int32)
    held, refs = torch.zeros(1, **ints), torch.zeros(4, **ints)
    for args in ((c.pool.cpu(), c.table, held.cuda(), refs.cuda()), (c.pool, c.table.cpu(), held.cuda(), refs.cuda()),
                 (c.pool, c.table, held, refs.cuda()), (c.pool, c.table, held.cuda(), refs)):
        with pytest.raises(ValueError):
            paged.PagePool(*args)
    for pool, table in ((c.pool.cpu(), c.table), (c.pool, c.table.cpu())):
        with pytest.raises(ValueError):
            paged.Kv4Cache(pool, table, n_q_heads=H, n_kv_heads=H, head_dim=D)
    with pytest.raises(ValueError):
        c.pages.copy(torch.zeros(1, **ints), torch.ones(1, **ints).cuda())
    with pytest.raises(ValueError):
        c.pages.compact(table_out=c.table.cpu())


def test_rope_calls():
    f, factor = native.rope_frequencies(D)
    table = torch.empty(8, D // 2, 2)
    with pytest.raises(ValueError):
        native.rope_table(f, table)
    t = table.cuda()
    native.rope_table(f, t, factor)
    x = torch.ones(3, H, D, device="cuda")
    pos = torch.zeros(3, dtype=torch.int32, device="cuda")
    for args, more in (((x.cpu(), None, x.cpu(), None, pos, t), {}), ((x, None, x, None, pos.cpu(), t), {}), ((x, None, x, None, pos, table), {}),
                       ((x, None, x, None, pos, t), {"q_gain": torch.ones(D)}), ((x, None, x, None, pos, t), {"status": torch.zeros(1, dtype=torch.int32)})):
        with pytest.raises(ValueError):
            native.rope_args(*args, **more)


def test_table_on_the_current_stream():
    f, _ = native.rope_frequencies(D)
    t = torch.zeros(4096, D // 2, 2, device="cuda")
    want = torch.zeros_like(t)
    native.rope_table(f, want)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        for _ in range(20):
            t.fill_(7.0)  # (a table filled on another stream would lose to one of these or to the copy)
            native.rope_table(f, t)
            got = t.clone()
            assert torch.equal(got, want)
