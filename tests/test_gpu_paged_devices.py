"""Calls whose tensors are not all on the pool's GPU, or that are made while another GPU is current, are refused before
anything is launched.  (A second GPU is pretended: get_device() and current_device() answer 1.)"""
import pytest
import torch

from paper_2609_26100_gb300 import native, paged

pytestmark = pytest.mark.gpu
H, D, N = 2, 128, 3


class Elsewhere(torch.Tensor):
    def get_device(self):
        return 1


def elsewhere(t):
    return t.as_subclass(Elsewhere)


@pytest.fixture
def cache():
    c = paged.Kv4Cache.allocate(n_layers=1, n_pages=4, n_seqs=2, max_pages=2, n_q_heads=H, n_kv_heads=H, head_dim=D)
    c.pages.reserve([0], [N])
    return c


def tensors():
    x = torch.ones(N, H, D, dtype=torch.bfloat16, device="cuda")
    return x, x.clone(), torch.zeros(N, dtype=torch.int32, device="cuda")


def calls(c):
    x, y, pos = tensors()
    b = c.batch([0], [0], [N])
    ids = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    table = torch.zeros(8, D // 2, 2, device="cuda")
    args = native.rope_args(x, None, y, None, pos, table)
    return [lambda **k: c.append(0, b, x, x, **k), lambda **k: c.read(0, b, x, y, **k), lambda **k: c.attention(0, b, x, y, **k),
            lambda **k: c.sync_status(**k), lambda **k: c.pages.reserve([1], [1], **k), lambda **k: c.pages.free([1], **k),
            lambda **k: c.pages.fork([0], [1], [N], **k), lambda **k: c.pages.compact(**k), lambda **k: c.pages.copy(*ids, **k),
            lambda **k: c.pages.sync_status(**k), lambda **k: native.qk_rope(args, **k),
            lambda **k: native.rope_table([1.0] * (D // 2), table, **k)]


@pytest.mark.parametrize("stream", [{}, {"stream": 0}])
def test_another_device_is_current(cache, monkeypatch, stream):
    every = calls(cache)
    torch.cuda.synchronize()
    state = [t.clone() for t in (cache.pool, cache.table, cache.pages.held, cache.pages.refs)]
    with monkeypatch.context() as m:
        m.setattr(torch.cuda, "current_device", lambda: 1)
        for call in every:
            with pytest.raises(ValueError):
                call(**stream)
    for a, b in zip(state, (cache.pool, cache.table, cache.pages.held, cache.pages.refs)):
        assert torch.equal(a, b)
    for call in every:  # (the same calls are taken where nothing is pretended)
        call(**stream)
    assert cache.sync_status() == native.TSS_OK and cache.pages.sync_status() == native.TSS_OK


def test_a_tensor_on_another_device(cache):
    c, b = cache, cache.batch([0], [0], [N])
    x, y, pos = tensors()
    lse, mask = torch.zeros(N, H, device="cuda"), torch.full((N, 2), -1, dtype=torch.int64, device="cuda")
    refused = [lambda: c.append(0, b, elsewhere(x), x), lambda: c.append(0, b, x, elsewhere(x)), lambda: c.read(0, b, elsewhere(x), y),
               lambda: c.read(0, b, None, elsewhere(y)), lambda: c.attention(0, b, elsewhere(x), y), lambda: c.attention(0, b, x, elsewhere(y)),
               lambda: c.attention(0, b, x, y, lse=elsewhere(lse)), lambda: c.attention(0, b, x, y, mask=elsewhere(mask)),
               lambda: c.attention(0, b, x, y, window=3, positions=elsewhere(pos)),
               lambda: c.pages.compact(table_out=elsewhere(c.table.clone())), lambda: c.pages.compact(refs_out=elsewhere(c.pages.refs.clone())),
               lambda: c.pages.copy(elsewhere(pos[:1].clone()), pos[1:2].clone()), lambda: c.pages.copy(pos[:1].clone(), elsewhere(pos[1:2].clone())),
               lambda: paged.PagePool(c.pool, elsewhere(c.table), c.pages.held, c.pages.refs),
               lambda: paged.PagePool(c.pool, c.table, elsewhere(c.pages.held), c.pages.refs),
               lambda: paged.PagePool(c.pool, c.table, c.pages.held, elsewhere(c.pages.refs)),
               lambda: paged.Kv4Cache(c.pool, elsewhere(c.table), n_q_heads=H, n_kv_heads=H, head_dim=D)]
    table = torch.zeros(8, D // 2, 2, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    refused += [lambda: native.rope_args(x, elsewhere(x), y, y, pos, table), lambda: native.rope_args(x, None, y, None, elsewhere(pos), table),
                lambda: native.rope_args(x, None, y, None, pos, elsewhere(table)),
                lambda: native.rope_args(x, None, y, None, pos, table, status=elsewhere(status)),
                lambda: native.rope_table([1.0] * (D // 2), elsewhere(table))]
    for i, call in enumerate(refused):
        with pytest.raises(ValueError):
            call()
            raise AssertionError(f"call {i} was taken")
    assert c.sync_status() == native.TSS_OK and c.pages.sync_status() == native.TSS_OK
