"""Reordering the page rows of sequences by parents on the device, against a plain restatement over Python lists."""
import random

import pytest
import torch

from paper_2609_26100_gb300 import native, paged

pytestmark = pytest.mark.gpu


def pool_of(n_seqs, max_pages, n_pages, rows, layers=2, elems=40):
    """A pool of distinct contents whose sequences hold the given pages."""
    pool = torch.arange(layers * n_pages * elems, dtype=torch.int32, device="cuda").view(layers, n_pages, elems)
    table = torch.full((n_seqs, max_pages), -1, dtype=torch.int32)
    refs = torch.zeros(n_pages, dtype=torch.int32)
    for s, row in enumerate(rows):
        table[s, :len(row)] = torch.tensor(row, dtype=torch.int32)
        for page in row:
            refs[page] += 1
    held = torch.tensor([len(r) for r in rows], dtype=torch.int32)
    return paged.PagePool(pool.clone(), table.cuda(), held.cuda(), refs.cuda())


def restated(p, seqs, parent, tokens):
    """(table, held, refs, pool) after the call."""
    table, held, refs, pool = p.table.cpu().clone(), p.held.tolist(), p.refs.tolist(), p.pool.cpu().clone()
    rows = [table[s, :held[s]].tolist() for s in range(len(held))]
    free = [i for i, r in enumerate(refs) if r == 0]
    new, copies = {}, []
    for i, s in enumerate(seqs):
        q = parent[i]
        if q < 0:
            new[s] = []
            continue
        full, total = tokens[q] // 64, -(-tokens[q] // 64)
        src = rows[seqs[q]][:total]
        takers = [j for j in range(len(seqs)) if parent[j] == q]
        keeper = q if q in takers else takers[0]
        if i != keeper:
            for x in range(full, total):
                page = free.pop(0)
                copies.append((src[x], page))
                src[x] = page
        new[s] = src
    for s, row in new.items():
        for page in rows[s]:
            refs[page] -= 1
        for page in row:
            refs[page] += 1
        table[s] = -1
        table[s, :len(row)] = torch.tensor(row, dtype=torch.int32)
        held[s] = len(row)
    before = pool.clone()
    for a, b in copies:
        pool[:, b] = before[:, a]
    return table, torch.tensor(held, dtype=torch.int32), torch.tensor(refs, dtype=torch.int32), pool


def check(p, seqs, parent, tokens):
    want = restated(p, seqs, parent, tokens)
    p.reorder(seqs, torch.tensor(parent, dtype=torch.int32, device="cuda"), tokens)
    for got, ref, what in zip((p.table, p.held, p.refs, p.pool), want, ("table", "held", "refs", "pool")):
        assert torch.equal(got.cpu(), ref), what
    assert p.sync_status() == native.TSS_OK


@pytest.mark.parametrize("seed", range(12))
def test_random_searches(seed):
    """Several selections in a row over beams of several texts, with pages reserved between them."""
    rng = random.Random(seed)
    groups = [rng.randrange(1, 9) for _ in range(rng.randrange(1, 5))]
    n = sum(groups)
    order = rng.sample(range(n + 3), n)          # other sequences stand between
    prefix = [rng.choice((0, 1, 3, 70, 131)) for _ in groups]
    max_pages = 150
    rows, ids = [[] for _ in range(n + 3)], iter(rng.sample(range(1200), 1200))
    tokens, at = [], 0
    for m, f in zip(groups, prefix):
        common = [next(ids) for _ in range(f)]
        for i in range(m):
            tokens.append(f * 64 + rng.choice((0, 1, 63, 64, 100, 130)) + (f == 0))
            rows[order[at]] = common + [next(ids) for _ in range(-(-tokens[-1] // 64) - f)] + [next(ids)] * (rng.random() < 0.3)
            at += 1
    for s in range(n + 3):
        if s not in order:
            rows[s] = [next(ids) for _ in range(2)]
    p = pool_of(n + 3, max_pages, 1200, rows)
    for _ in range(3):
        parent, base = [], 0
        for m in groups:
            parent += [base + rng.randrange(m) if rng.random() < 0.9 else -1 for _ in range(m)]
            base += m
        check(p, order, parent, tokens)
        tokens = [tokens[q] if q >= 0 else 0 for q in parent]
        tokens = [t + 1 if t else 0 for t in tokens]
        p.reserve(order, tokens)


@pytest.mark.parametrize("parent", [[0, 1, 2, 3], [1, 0, 3, 2], [1, 2, 3, 0], [3, 3, 3, 3], [2, 2, 0, 0], [-1, -1, -1, -1], [-1, 0, 0, -1]])
@pytest.mark.parametrize("tokens", [[1, 1, 1, 1], [64, 64, 64, 64], [65, 100, 128, 640], [0, 0, 0, 0]])
def test_permutations(parent, tokens):
    ids = iter(range(5, 100))
    rows = [[next(ids) for _ in range(-(-t // 64))] for t in tokens]
    check(pool_of(4, 12, 100, rows), [0, 1, 2, 3], parent, tokens)


def test_64_beams_of_a_long_text():
    rng = random.Random(1)
    common = rng.sample(range(4000), 700)
    rest = [i for i in range(4000) if i not in set(common)]
    rows = [common + [rest.pop() for _ in range(3)] for _ in range(64)]
    tokens = [700 * 64 + 130 + i for i in range(62)] + [700 * 64 + 192] * 2
    p = pool_of(64, 1024, 4000, rows, layers=3, elems=4100)
    check(p, list(range(64)), [rng.randrange(64) for _ in range(64)], tokens)


def test_what_the_device_refuses():
    rows = [[4, 5, 6], [4, 7], [8]]
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731

    def unchanged(p, seqs, parent, tokens, status):
        before = [x.clone() for x in (p.table, p.held, p.refs, p.pool)]
        p.reorder(seqs, parent, tokens)
        assert p.sync_status() == status and p.sync_status() == native.TSS_OK
        assert all(torch.equal(a, b) for a, b in zip(before, (p.table, p.held, p.refs, p.pool)))

    # no free page for the copies
    p = pool_of(3, 4, 9, rows)
    p.refs[:4] = 1
    unchanged(p, [0, 1], i32(0, 0), [130, 70], native.TSS_ERR_KV_CAPACITY)
    p = pool_of(3, 4, 12, rows)
    unchanged(p, [0, 1], i32(0, 2), [130, 70], native.TSS_ERR_DEVICE_CHECK)     # no such entry
    unchanged(p, [0, 1], i32(-2, 0), [130, 70], native.TSS_ERR_DEVICE_CHECK)
    unchanged(p, [0, 1], i32(1, 1), [130, 129], native.TSS_ERR_DEVICE_CHECK)    # the parent holds less
    p.held[1] = 5                                                              # more than the table has
    unchanged(p, [0, 1], i32(0, 0), [130, 70], native.TSS_ERR_DEVICE_CHECK)
    p = pool_of(3, 4, 12, rows)
    p.table[0, 2] = 12                                                         # a page to copy that is none
    unchanged(p, [0, 1], i32(0, 0), [130, 70], native.TSS_ERR_DEVICE_CHECK)
    # the parent's length counts only where somebody goes on with it
    check(pool_of(3, 4, 12, rows), [0, 1], [0, 0], [130, 200])
    # an id outside the pool in a shared place moves as it is
    p = pool_of(3, 4, 12, rows)
    p.table[0, 0] = 99
    p.reorder([0, 1], i32(0, 0), [130, 70])
    assert p.sync_status() == native.TSS_ERR_DEVICE_CHECK
    assert p.table[:2, :3].tolist() == [[99, 5, 6], [99, 5, 0]] and p.refs[[4, 5, 6, 7, 0]].tolist() == [1, 2, 1, 0, 1]


def test_refusals():
    p = pool_of(3, 4, 12, [[4, 5, 6], [4, 7], [8]])
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731

    def refused(*a):
        with pytest.raises((native.TssError, ValueError)):
            p.reorder(*a)

    refused([0, 0], i32(0, 1), [1, 1])
    refused([0, 3], i32(0, 1), [1, 1])
    refused([0, -1], i32(0, 1), [1, 1])
    refused([0, 1], i32(0, 1, 1), [1, 1])
    refused([0, 1], i32(0, 1), [1])
    refused([0, 1], i32(0, 1), [1, -1])
    refused([0, 1], i32(0, 1), [1, 257])
    refused([0, 1], i32(0, 1).long(), [1, 1])
    refused([0, 1], i32(0, 1).cpu(), [1, 1])
    refused(list(range(65)), torch.zeros(65, dtype=torch.int32, device="cuda"), [1] * 65)
    p.reorder([], i32(), [])
    assert p.sync_status() == native.TSS_OK


def test_captured_with_parents_of_another_launch():
    rows = [[4, 5], [4, 6], [4, 7]]
    p = pool_of(3, 4, 20, rows)
    parent = torch.zeros(3, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.reorder([0, 1, 2], parent, [100, 100, 100])
    for now in ([0, 0, 2], [1, 2, 0], [2, 2, 2]):
        want = restated(p, [0, 1, 2], now, [100] * 3)
        parent.copy_(torch.tensor(now, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a.cpu(), b) for a, b in zip((p.table, p.held, p.refs, p.pool), want))
    assert p.sync_status() == native.TSS_OK
