"""tss_pages_*: reserving, freeing, forking, compacting and copying pages, against a model in Python.
Everything is whole numbers and moved bytes: compared for equality."""
import random

import pytest
import torch

from paper_2609_26100_gb300 import native, paged

pytestmark = pytest.mark.gpu


class Model:
    """The same books on the host; `data` names the content of each page."""

    def __init__(self, n_seqs, max_pages, n_pages):
        self.rows = [[] for _ in range(n_seqs)]
        self.refs, self.max_pages = [0] * n_pages, max_pages
        self.data = list(range(n_pages))

    def lowest(self, n):
        return [i for i, r in enumerate(self.refs) if r == 0][:n]

    def reserve(self, seqs, pages):
        need = sum(max(0, p - len(self.rows[s])) for s, p in zip(seqs, pages))
        free = self.lowest(need)
        if len(free) < need:
            return False
        for s, p in zip(seqs, pages):
            while len(self.rows[s]) < p:
                i = free.pop(0)
                self.refs[i] = 1
                self.rows[s].append(i)
        return True

    def free(self, seqs, keep):
        for s, k in zip(seqs, keep):
            for i in self.rows[s][k:]:
                self.refs[i] -= 1
            self.rows[s] = self.rows[s][:k]

    def fork(self, src, dst, tokens):
        need = sum(t % 64 > 0 for t in tokens)
        free = self.lowest(need)
        if len(free) < need:
            return False
        for s, d, t in zip(src, dst, tokens):
            self.rows[d] = self.rows[s][:t // 64]
            for i in self.rows[d]:
                self.refs[i] += 1
            if t % 64:
                i = free.pop(0)
                self.refs[i] = 1
                self.data[i] = self.data[self.rows[s][t // 64]]
                self.rows[d].append(i)
        return True

    def compact(self):
        n = sum(r > 0 for r in self.refs)
        move = dict(zip([i for i in range(n, len(self.refs)) if self.refs[i] > 0], [i for i in range(n) if self.refs[i] == 0]))
        for a, b in move.items():
            self.refs[b], self.refs[a] = self.refs[a], 0
            self.data[b] = self.data[a]
        self.rows = [[move.get(i, i) for i in row] for row in self.rows]

    def table(self):
        return torch.tensor([row + [-1] * (self.max_pages - len(row)) for row in self.rows], dtype=torch.int32)


def make(n_seqs, max_pages, n_pages, layers=2, elems=24):
    pool = (torch.arange(n_pages, device="cuda")[None, :, None] * 7 + torch.arange(layers, device="cuda")[:, None, None] * 100003
            + torch.arange(elems, device="cuda") * 13).to(torch.int32)
    pages = paged.PagePool(pool.clone(), torch.full((n_seqs, max_pages), -1, dtype=torch.int32, device="cuda"),
                           torch.zeros(n_seqs, dtype=torch.int32, device="cuda"), torch.zeros(n_pages, dtype=torch.int32, device="cuda"))
    return pages, Model(n_seqs, max_pages, n_pages), pool


def same(pages, model, pool):
    assert torch.equal(pages.table.cpu(), model.table())
    assert pages.held.tolist() == [len(r) for r in model.rows]
    assert pages.refs.tolist() == model.refs
    assert torch.equal(pages.pool, pool[:, torch.tensor(model.data, device="cuda")])


@pytest.mark.parametrize("seed,n_pages,elems", [(0, 40, 24), (1, 200, 4), (2, 97, 9000), (3, 33, 4096 * 3 + 4)])
def test_random_histories(seed, n_pages, elems):
    rng = random.Random(seed)
    pages, model, pool = make(12, 20, n_pages, elems=elems)
    ok = 0
    for step in range(60):
        kind = rng.choice(("reserve", "reserve", "fork", "fork", "free", "compact"))
        if kind == "reserve":
            seqs = rng.sample(range(12), rng.randrange(1, 5))
            tokens = [rng.randrange(0, 64 * 8) for _ in seqs]
            pages.reserve(seqs, tokens)
            good = model.reserve(seqs, [-(-t // 64) for t in tokens])
        elif kind == "free":
            seqs = rng.sample(range(12), rng.randrange(1, 6))
            if rng.random() < 0.5:
                pages.free(seqs)
                model.free(seqs, [0] * len(seqs))
            else:
                keep = [rng.randrange(0, 64 * 9) for _ in seqs]
                pages.free(seqs, keep)
                model.free(seqs, [-(-t // 64) for t in keep])
            good = True
        elif kind == "fork":
            dst = [s for s in range(12) if not model.rows[s]][:rng.randrange(1, 5)]
            src = [s for s in range(12) if model.rows[s]]
            if not dst or not src:
                continue
            src = [rng.choice(src) for _ in dst]
            tokens = [rng.randrange(0, 64 * len(model.rows[s]) + 1) for s in src]
            pages.fork(src, dst, tokens)
            good = model.fork(src, dst, tokens)
        else:
            pages.compact()
            model.compact()
            good = True
        assert pages.sync_status() == (native.TSS_OK if good else native.TSS_ERR_KV_CAPACITY)
        ok += good
        same(pages, model, pool)
    assert ok > 30


def test_large_pools_and_the_last_pages():
    """More pages than one round of the search, nearly all taken; and the largest pool's books."""
    for n in (16384, 16385, 50000, 1 << 20):
        pages, _, _ = make(4, 70, n, layers=1, elems=4)
        pages.refs[:] = 1
        free = sorted(random.Random(n).sample(range(n), 60) + [n - 1, n - 2, 0])
        free = sorted(set(free))
        pages.refs[torch.tensor(free, device="cuda")] = 0
        pages.reserve([2, 0], [64 * 20, 64 * (len(free) - 20)])
        assert pages.sync_status() == native.TSS_OK
        assert pages.table[2, :20].tolist() == free[:20] and pages.table[0, :len(free) - 20].tolist() == free[20:]
        assert (pages.refs == 1).all()
        pages.reserve([1], [1])
        assert pages.sync_status() == native.TSS_ERR_KV_CAPACITY and int(pages.held[1]) == 0
        # thin the pool out and make it dense again
        live = torch.zeros(n, dtype=torch.bool)
        live[torch.randperm(n, generator=torch.Generator().manual_seed(n))[:n // 3]] = True
        pages.refs[:] = live.to(torch.int32).cuda() * 3
        pages.table[:] = -1
        some = live.nonzero()[:, 0][-70:].to(torch.int32).cuda()
        pages.table[3] = some
        was = pages.pool.clone()
        pages.compact()
        assert pages.sync_status() == native.TSS_OK
        L = int(live.sum())
        assert (pages.refs[:L] == 3).all() and (pages.refs[L:] == 0).all()
        assert torch.equal(pages.pool[0, pages.table[3].long()], was[0, some.long()])
        pages.close()


def test_compact_out_of_place_leaves_the_books():
    pages, model, pool = make(4, 8, 30)
    pages.reserve([0, 1, 2], [64 * 8, 64 * 7, 64 * 8])
    model.reserve([0, 1, 2], [8, 7, 8])
    pages.free([0])
    model.free([0], [0])
    same(pages, model, pool)
    before = [x.clone() for x in (pages.table, pages.refs, pages.held)]
    t, r = torch.full_like(pages.table, 99), torch.full_like(pages.refs, 99)
    for _ in range(2):  # (the pages that moved still hold their bytes: again gives the same)
        pages.compact(t, r)
        for x, y in zip((pages.table, pages.refs, pages.held), before):
            assert torch.equal(x, y)
        m = Model(4, 8, 30)
        m.rows, m.refs, m.data = [list(x) for x in model.rows], list(model.refs), list(model.data)
        m.compact()
        assert torch.equal(t.cpu(), m.table()) and r.tolist() == m.refs
        assert torch.equal(pages.pool, pool[:, torch.tensor(m.data, device="cuda")])


def test_copy():
    pages, _, pool = make(2, 4, 20, layers=3, elems=8192)
    src, dst = torch.tensor([3, 3, 19], dtype=torch.int32, device="cuda"), torch.tensor([0, 7, 1], dtype=torch.int32, device="cuda")
    pages.copy(src, dst)
    want = pool.clone()
    want[:, dst.long()] = pool[:, src.long()]
    assert torch.equal(pages.pool, want) and pages.sync_status() == native.TSS_OK
    pages.copy(torch.tensor([20, -1, 4, 5], dtype=torch.int32, device="cuda"), torch.tensor([2, 2, 20, 6], dtype=torch.int32, device="cuda"))
    want[:, 6] = pool[:, 5]
    assert torch.equal(pages.pool, want) and pages.sync_status() == native.TSS_ERR_DEVICE_CHECK
    pages.copy(src[:0], dst[:0])


def test_contradicting_books_are_recorded_and_left():
    def books(p):
        return [x.clone() for x in (p.table, p.held, p.refs, p.pool)]

    pages, _, _ = make(4, 8, 20)
    pages.reserve([0, 1], [200, 100])
    was = books(pages)
    for src, dst, tokens in (([0], [1], [64]), ([0], [2], [64 * 5]), ([3], [2], [1])):  # dst in use; src too short, empty
        pages.fork(src, dst, tokens)
        assert pages.sync_status() == native.TSS_ERR_DEVICE_CHECK
        assert all(torch.equal(a, b) for a, b in zip(was, books(pages)))
    pages.table[0, 0] = 20  # no page of the pool
    was = books(pages)
    pages.fork([0], [2], [64])
    assert pages.sync_status() == native.TSS_ERR_DEVICE_CHECK
    assert all(torch.equal(a, b) for a, b in zip(was, books(pages)))
    pages.held[3] = -1
    pages.reserve([3], [1])
    assert pages.sync_status() == native.TSS_ERR_DEVICE_CHECK
    refs = pages.refs.clone()
    held = [int(x) for x in pages.table[0, 1:4]]
    pages.free([0])  # the entry that names no page is dropped, the others are given back
    assert pages.sync_status() == native.TSS_ERR_DEVICE_CHECK
    refs[torch.tensor(held, device="cuda")] -= 1
    assert torch.equal(pages.refs, refs) and (pages.table[0] == -1).all() and int(pages.held[0]) == 0


def test_refusals():
    pages, _, _ = make(4, 8, 20)

    def status(call, *a):
        with pytest.raises(native.TssError) as e:
            call(*a)
        return e.value.status

    bad, cap = native.TSS_ERR_INVALID_ARG, native.TSS_ERR_KV_CAPACITY
    assert status(pages.reserve, [4], [1]) == bad
    assert status(pages.reserve, [-1], [1]) == bad
    assert status(pages.reserve, [1, 1], [1, 1]) == bad
    assert status(pages.reserve, [1], [-65]) == bad
    assert status(pages.reserve, [1], [64 * 9]) == cap
    assert status(pages.free, [0, 0]) == bad
    assert status(pages.free, [0], [-64]) == bad
    assert status(pages.free, list(range(4)) * 17) == bad
    assert status(pages.fork, [0], [0], [1]) == bad
    assert status(pages.fork, [0, 1], [1, 2], [1, 1]) == bad
    assert status(pages.fork, [0, 1], [2, 2], [1, 1]) == bad
    assert status(pages.fork, [0], [1], [64 * 9]) == cap
    assert status(pages.fork, [0], [1], [-65]) == bad
    with pytest.raises(ValueError):
        pages.reserve([0], [1, 2])
    with pytest.raises(ValueError):
        pages.compact(pages.table[:2])
    pages.reserve([], [])
    pages.free([])
    pages.fork([], [], [])
    assert pages.sync_status() == native.TSS_OK and (pages.refs == 0).all()


@pytest.mark.parametrize("shape", [(0, 1, 1), (1, 0, 1), (1, 1, 0), (1, 1, (1 << 20) + 1), (1 << 16, 1 << 16, 4)])
def test_create_refusals(shape):
    import ctypes
    h = ctypes.c_void_p()
    assert native.lib().tss_pages_create(*shape, ctypes.byref(h)) == native.TSS_ERR_INVALID_ARG and not h.value
