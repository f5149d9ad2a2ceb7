"""Attention of sequences that share the pages of a prefix, against the definition in 64 bits on the values held, request by
request.

Tolerances.  The output's half step (eps / 2 of it).  Weights of one fp16 part, bf16 outputs where some request or group of the call
has more than 8 rows of a KV head: of v = s c + z the sum of p s c takes p s rounded by up to 2^-12 of it, while that of p z does not,
so the output is off by up to 2^-12 of the mean of s c = v - z.  As z is the least value of its group, that is at most the
largest value less the smallest, twice the largest magnitude.  Scores and sums in fp32: a score's error of 2^-20 of the largest
score's size or one moves the weights by as much, and with them the output by that share of the largest value, twice."""
import math
import random

import pytest
import torch

import paged_ref as R
from paper_2609_26100_gb300 import native, paged

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


def shared_cache(sizes, shared, first, n, hq, hk, d, seed=0, room=None, poison=0xFF):
    """Sequences in groups whose whole pages of the first shared[g] tokens are the same ones; every token appended.  What is not is
    NaN.  (cache, k, v): values held, [seq] -> [tokens][hk][d] in 64 bits."""
    total = [f + m for f, m in zip(first, n)]
    gen = random.Random(seed)
    need = sum(s // 64 for s in shared) + sum(-(-t // 64) + 1 for t in total)
    ids = iter(gen.sample(range(need + 2), need + 2))
    table, at = torch.full((len(total), max(-(-t // 64) for t in total) + 1), -1, dtype=torch.int32), 0
    for g, m in enumerate(sizes):
        common = [next(ids) for _ in range(shared[g] // 64)]
        for b in range(at, at + m):
            own = -(-total[b] // 64) - len(common)
            row = common[:-(-total[b] // 64)] + [next(ids) for _ in range(own)]
            table[b, :len(row)] = torch.tensor(row, dtype=torch.int32)
        at += m
    pool = torch.full((1, need + 2, paged.page_bytes(hk, d)), poison, dtype=torch.uint8, device="cuda")
    c = paged.Kv4Cache(pool, table.cuda(), n_q_heads=hq, n_kv_heads=hk, head_dim=d, shared_rows=sum(n) if room is None else room)
    rnd = torch.Generator(device="cuda").manual_seed(seed + 1)
    at = 0
    for g, m in enumerate(sizes):
        for b in range(at, at + m):
            start = shared[g] // 64 * 64 if b > at else 0
            k, v = (torch.randn(total[b] - start, hk, d, generator=rnd, device="cuda").to(BF) for _ in range(2))
            if total[b] > start:
                c.append(0, c.batch([b], [start], [total[b] - start]), k, v)
        at += m
    held = [[R.sequence_values(c.pool[0], c.table, b, t, hk, d, side) for b, t in enumerate(total)] for side in (0, 1)]
    return c, *held


def reference(k, v, q, see, scale):
    n, hq, d = q.shape
    g = hq // k.shape[1]
    k, v = (torch.nan_to_num(x).repeat_interleave(g, 1) for x in (k, v))  # (what nobody sees may be NaN)
    s = (torch.einsum("nhd,shd->nhs", q, k) * scale).masked_fill(~see[:, None], -math.inf)
    lse = torch.logsumexp(s, -1)
    w = torch.where(torch.isinf(lse)[..., None], 0.0, (s - torch.where(torch.isinf(lse), 0.0, lse)[..., None]).exp())
    size = torch.where(see[:, None], s, 0.0).abs().amax()
    return torch.einsum("nhs,shd->nhd", w, v), lse, size


def run_and_check(c, k, v, sizes, shared, first, n, *, dtype=BF, window=0, sinks=0, masks=None, positions=None, seed=5, scale=None, call=None):
    hq, d = c.n_q_heads, c.head_dim
    gq = hq // c.n_kv_heads
    rnd = torch.Generator(device="cuda").manual_seed(seed)
    q = (torch.randn(sum(n), hq, d, generator=rnd, device="cuda") * 1.5).to(dtype)
    out = torch.full((sum(n) + 1, hq, d), 7.0, dtype=dtype, device="cuda")
    lse = torch.full((sum(n) + 1, hq), 7.0, device="cuda")
    words = torch.tensor(R.words([x for m in masks for x in m]), dtype=torch.int64, device="cuda") if masks else None
    pos = torch.tensor([x for p in positions for x in p], dtype=torch.int32, device="cuda") if positions else None
    batch, groups = c.batch(list(range(len(n))), first, n), c.groups(sizes, shared)
    c.attention_shared(0, batch, groups, q, out[:-1], lse=lse[:-1], window=window, sinks=sinks, mask=words, positions=pos, scale=scale)
    assert c.sync_status() == native.TSS_OK
    assert (out[-1] == 7.0).all() and (lse[-1] == 7.0).all()  # rows behind the last stay as they were
    rows, at = [], 0
    for m in sizes:
        rows += [sum(n[at:at + m])] + n[at:at + m]
        at += m
    one_part = 2.0 ** -11 if dtype == BF and max(rows) * gq > 8 else 0.0
    at = 0
    for b, m in enumerate(n):
        if m == 0:
            continue
        see = R.sees(first[b], m, masks[b] if masks else None, positions[b] if positions else range(first[b], first[b] + m), window, sinks, "cuda")
        ref, ref_lse, size = reference(k[b], v[b], q[at:at + m].double(), see, d ** -0.5 if scale is None else scale)
        vmax = torch.nan_to_num(v[b]).abs().amax()
        room = ref.abs() * torch.finfo(dtype).eps / 2 + vmax * (one_part + (1 + size) * 2.0 ** -19)
        got = out[at:at + m].double()
        lost = (see & torch.isnan(v[b]).any(-1).any(-1)).any(-1)  # (rows that see a NaN: NaN)
        assert torch.isnan(got[lost]).all() and torch.isnan(lse[at:at + m][lost]).all()
        got, ref = got.masked_fill(lost[:, None, None], 0.0), ref.masked_fill(lost[:, None, None], 0.0)
        lse[at:at + m][lost], ref_lse[lost] = 0.0, 0.0
        assert ((got - ref).abs() <= room).all(), (b, float(((got - ref).abs() - room).max()))
        inf = torch.isinf(ref_lse)
        assert torch.equal(inf, torch.isinf(lse[at:at + m]))
        assert (torch.where(inf, 0.0, lse[at:at + m].double() - ref_lse).abs() <= 2e-5 * (1 + size)).all()
        at += m
    return q, out[:-1], lse[:-1]


CASES = [  # sizes, shared, extra context of each, rows of each, hq, hk, d, dtype
    ((2,), (64,), (0, 0), (1, 1), 2, 2, 128, BF),
    ((3,), (0,), (5, 70, 0), (1, 1, 2), 4, 2, 128, HF),
    ((3,), (63,), (5, 70, 0), (1, 1, 2), 4, 2, 64, BF),
    ((4,), (1000,), (0, 1, 40, 200), (1, 1, 1, 1), 2, 2, 128, BF),
    ((8,), (130,), (0, 1, 40, 64, 62, 63, 7, 300), (1,) * 8, 4, 4, 64, HF),
    ((9,), (2050,), (3,) * 9, (1,) * 9, 2, 2, 128, HF),
    ((2, 1, 3), (300, 65, 128), (1, 2, 3, 4, 5, 6), (1, 2, 3, 0, 5, 1), 8, 2, 128, BF),
    ((3, 2), (640, 500), (0, 10, 20, 30, 40), (0, 0, 4, 7, 0), 4, 2, 128, BF),
    ((5,), (4000,), (17,) * 5, (6,) * 5, 8, 2, 128, BF),        # 120 rows of a KV head: one tile of 128
    ((4,), (900,), (17, 0, 5, 64), (61, 33, 61, 60), 4, 2, 128, HF),  # 430 rows, and own blocks of more than 48
    ((4,), (900,), (17, 0, 5, 64), (61, 33, 61, 60), 4, 2, 128, BF),
    ((3,), (700,), (9, 9, 130), (128, 1, 128), 1, 1, 128, BF),
    ((6,), (700,), (9,) * 6, (20,) * 6, 4, 2, 64, HF),          # many rows at head_dim 64
    ((64,), (257,), (2,) * 64, (1,) * 64, 1, 1, 128, BF),
    ((1, 1), (256, 320), (3, 4), (2, 1), 4, 4, 128, HF),        # no one to share with
]


@pytest.mark.parametrize("sizes,shared,extra,n,hq,hk,d,dtype", CASES)
def test_chains(sizes, shared, extra, n, hq, hk, d, dtype):
    group = [g for g, m in enumerate(sizes) for _ in range(m)]
    first = [shared[g] + e for g, e in zip(group, extra)]
    c, k, v = shared_cache(sizes, shared, first, list(n), hq, hk, d)
    run_and_check(c, k, v, list(sizes), list(shared), first, list(n), dtype=dtype)


@pytest.mark.parametrize("window,sinks", [(1, 0), (40, 3), (300, 0), (300, 70), (900, 4), (5000, 5), (100, 2000), (64, 640), (50, 641), (2 ** 31 - 1, 0)])
@pytest.mark.parametrize("n", [(1, 1, 1), (9, 4, 33)])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_windows(window, sinks, n, dtype):
    """Windows that leave out the shared keys, some of them, or none, for requests of other lengths; first tokens that reach past
    the shared part."""
    sizes, shared, first = [3], [700], [700, 1100, 903]
    c, k, v = shared_cache(sizes, shared, first, list(n), 4, 2, 128, seed=3)
    run_and_check(c, k, v, sizes, shared, first, list(n), dtype=dtype, window=window, sinks=sinks)


@pytest.mark.parametrize("d,hq", [(128, 4), (64, 4), (128, 16)])
@pytest.mark.parametrize("window", [0, 350])
def test_trees_with_positions_and_empty_rows(d, hq, window):
    rng = random.Random(d + hq)
    sizes, shared, n = [2, 3], [448, 64], [17, 5, 1, 40, 9]
    first = [450, 600, 64, 100, 333]
    masks = [[(1 << i) | rng.getrandbits(i) if i else 1 for i in range(m)] for m in n]
    masks[3][7] = 0                                # (sees no row of its block)
    positions = [[f + rng.randrange(m) for _ in range(m)] for f, m in zip(first, n)]
    positions[0][3] = 2                            # below the context's end: counts as its end
    c, k, v = shared_cache(sizes, shared, first, n, hq, 2, d, seed=4)
    run_and_check(c, k, v, sizes, shared, first, n, masks=masks, positions=positions, window=window, sinks=2 if window else 0)


def test_rows_that_see_nothing():
    sizes, shared, first, n = [2], [256], [256, 320], [3, 60]
    masks = [[0] * m for m in n]
    c, k, v = shared_cache(sizes, shared, first, n, 2, 1, 128, seed=6)
    for positions in ([[2 ** 31 - 1] * m for m in n], [[f] * m for f, m in zip(first, n)]):
        run_and_check(c, k, v, sizes, shared, first, n, masks=masks, positions=positions, window=1)


def test_nan_in_unseen_pages():
    """Pages before the window, shared and own, that hold NaN; and NaN that is seen stays NaN (a window of 200 before token 900 sees
    keys 701 .. 703 of the own page that holds it; the other two requests see none)."""
    sizes, shared, first, n = [3], [640], [640, 900, 700], [1, 2, 1]
    c, k, v = shared_cache(sizes, shared, first, n, 4, 2, 128, seed=7)
    c.pool[0, c.table[0, :6].long()] = 0xFF
    c.pool[0, c.table[1, 10].long()] = 0xFF
    k, v = ([R.sequence_values(c.pool[0], c.table, b, f + m, 2, 128, side) for b, (f, m) in enumerate(zip(first, n))] for side in (0, 1))
    q, out, lse = run_and_check(c, k, v, sizes, shared, first, n, window=200)
    assert torch.isfinite(out[[0, 3]].float()).all()
    # without that page NaN is nowhere in sight
    run_and_check(c, k, v, sizes, shared, first, n, window=196)
    c.attention_shared(0, c.batch([0, 1, 2], first, n), c.groups(sizes, shared), q, out)
    assert torch.isnan(out.float()).all()


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("spread", [1e-3, 30.0])
def test_flat_and_steep_scores(dtype, spread):
    sizes, shared, n = [20], [3000], [1] * 20
    first = [3000 + 31 * i for i in range(20)]
    c, k, v = shared_cache(sizes, shared, first, n, 4, 1, 128, seed=8)
    run_and_check(c, k, v, sizes, shared, first, n, dtype=dtype, scale=spread * 128 ** -0.5)


@pytest.mark.parametrize("rows", [9, 16, 31, 33, 64, 65, 80, 97, 128, 129, 200])
@pytest.mark.parametrize("tokens", [64, 128, 192, 1088])
def test_row_counts(rows, tokens):
    """Numbers of rows around the kernels' blocks, over few pages and some."""
    m = min(rows, 64)
    n = [rows // m + (i < rows % m) for i in range(m)]
    c, k, v = shared_cache([m], [tokens], [tokens] * m, n, 2, 2, 128, seed=rows)
    run_and_check(c, k, v, [m], [tokens], [tokens] * m, n)


@pytest.mark.parametrize("size", [1e-7, 1e-3, 300.0, 2e4, 6e4, 3e5])
@pytest.mark.parametrize("rows", [12, 90])
def test_magnitudes_of_values(size, rows):
    """Values over the whole range that pages hold, a few tokens much larger than the rest."""
    first, n = [330, 320], [rows // 2, rows // 2]
    c, k, v = shared_cache([2], [320], first, n, 2, 2, 128, seed=20)
    g = torch.Generator(device="cuda").manual_seed(21)
    kk = torch.randn(320, 2, 128, generator=g, device="cuda").to(BF)
    vv = torch.randn(320, 2, 128, generator=g, device="cuda") * min(size, 1.0)
    vv[::7] *= max(size, 1.0)
    c.append(0, c.batch([0], [0], [320]), kk, vv.to(BF))
    k, v = ([R.sequence_values(c.pool[0], c.table, b, f + m, 2, 128, side) for b, (f, m) in enumerate(zip(first, n))] for side in (0, 1))
    run_and_check(c, k, v, [2], [320], first, n, scale=0.02)


def test_scores_that_rise_page_by_page():
    """Keys ever nearer to the queries: references rise at nearly every tile, the outputs so far are scaled each time."""
    for rows in (16, 100):
        first, n = [2048, 2048], [rows // 2, rows // 2]
        c, k, v = shared_cache([2], [2048], first, n, 2, 2, 128, seed=22)
        g = torch.Generator(device="cuda").manual_seed(23)
        kk = torch.randn(1, 2, 128, generator=g, device="cuda") * torch.linspace(-3, 3, 2048, device="cuda")[:, None, None]
        vv = torch.randn(2048, 2, 128, generator=g, device="cuda")
        c.append(0, c.batch([0], [0], [2048]), kk.to(BF), vv.to(BF))
        k, v = ([R.sequence_values(c.pool[0], c.table, b, f + m, 2, 128, side) for b, (f, m) in enumerate(zip(first, n))] for side in (0, 1))
        run_and_check(c, k, v, [2], [2048], first, n, scale=0.5)


@pytest.mark.parametrize("d,n,dtype", [(128, 1, BF), (64, 1, HF), (64, 9, HF), (128, 9, BF)])
@pytest.mark.parametrize("window", [0, 130])
def test_more_items_of_own_keys_than_warps(d, n, dtype, window):
    """64 requests of 32 heads: more items of few keys than warps that run at a time."""
    rng = random.Random(d + n)
    first = [64 + rng.randrange(260) for _ in range(64)]
    c, k, v = shared_cache([64], [64], first, [n] * 64, 32, 32, d, seed=15)
    run_and_check(c, k, v, [64], [64], first, [n] * 64, dtype=dtype, window=window, sinks=3 if window else 0)


def test_as_the_attention_of_each():
    """The same as tss_paged_attention, up to the weights' bits and the order of sums; and twice the same bits."""
    sizes, shared, n = [12, 5], [1500, 777], [1] * 17
    first = [s + 13 * i for m, s in zip(sizes, shared) for i in range(m)]
    c, k, v = shared_cache(sizes, shared, first, n, 8, 2, 128, seed=9)
    q, out, lse = run_and_check(c, k, v, sizes, shared, first, n, dtype=HF)
    batch, groups = c.batch(list(range(17)), first, n), c.groups(sizes, shared)
    one, one_lse, again = torch.empty_like(out), torch.empty_like(lse), torch.empty_like(out)
    c.attention(0, batch, q, one, lse=one_lse)
    c.attention_shared(0, batch, groups, q, again)
    assert torch.equal(out, again)
    assert ((out.float() - one.float()).abs() <= one.float().abs() * 2.0 ** -10 + 2.0 ** -15).all()
    assert ((lse - one_lse).abs() <= 1e-5 * (1 + one_lse.abs())).all()
    # a batch whose groups are single requests is the attention of each, bit for bit
    c.attention_shared(0, batch, c.groups([1] * 17, [0] * 17), q, again)
    assert torch.equal(again, one)


def test_strides_streams_and_graphs():
    sizes, shared, first, n = [4], [1000], [1000, 1010, 1100, 1064], [1, 1, 1, 1]
    c, k, v = shared_cache(sizes, shared, first, n, 4, 2, 128, seed=10)
    q, out, lse = run_and_check(c, k, v, sizes, shared, first, n)
    batch, groups = c.batch([0, 1, 2, 3], first, n), c.groups(sizes, shared)
    wide, wide_out = (torch.zeros(4, 7, 128, dtype=BF, device="cuda") for _ in range(2))
    wide[:, 1:5] = q
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        c.attention_shared(0, batch, groups, wide[:, 1:5], wide_out[:, 2:6])
    side.synchronize()
    assert torch.equal(wide_out[:, 2:6], out) and (wide_out[:, :2] == 0).all() and (wide_out[:, 6:] == 0).all()
    graph = torch.cuda.CUDAGraph()
    mine, got = q.clone(), torch.empty_like(out)
    with torch.cuda.graph(graph):
        c.attention_shared(0, batch, groups, mine, got)
    mine.copy_(q.flip(0))
    graph.replay()
    want = torch.empty_like(out)
    c.attention_shared(0, batch, groups, q.flip(0).contiguous(), want)
    assert torch.equal(got, want)


def test_pages_that_are_missing():
    sizes, shared, first, n = [2], [256], [300, 256], [1, 1]
    c, k, v = shared_cache(sizes, shared, first, n, 2, 2, 128, seed=11)
    q = torch.randn(2, 2, 128, device="cuda").to(BF)
    out = torch.empty_like(q)
    c.table[0, 1] = -1
    c.attention_shared(0, c.batch([0, 1], first, n), c.groups(sizes, shared), q, out)
    assert c.sync_status() == native.TSS_ERR_DEVICE_CHECK and torch.isfinite(out.float()).all()


@pytest.mark.parametrize("rows", [1, 40])
def test_a_wait_that_runs_out(rows):
    sizes, shared, first, n = [2], [256], [256, 256], [rows, rows]
    c, k, v = shared_cache(sizes, shared, first, n, 2, 2, 128, seed=12)
    c.inject_timeout(1)
    q = torch.randn(2 * rows, 2, 128, device="cuda").to(BF)
    c.attention_shared(0, c.batch([0, 1], first, n), c.groups(sizes, shared), q, torch.empty_like(q))
    assert c.sync_status() == native.TSS_ERR_TIMEOUT
    run_and_check(c, k, v, sizes, shared, first, n)


def test_refusals():
    sizes, shared, first, n = [2, 1], [128, 64], [130, 128, 64], [2, 1, 1]
    c, k, v = shared_cache(sizes, shared, first, n, 2, 2, 128, seed=13, room=4)
    q = torch.zeros(4, 2, 128, dtype=BF, device="cuda")
    out = torch.empty_like(q)
    batch = c.batch([0, 1, 2], first, n)

    def refused(b, *groups, x=q):
        with pytest.raises((native.TssError, ValueError)):
            c.attention_shared(0, b, c.groups(*groups), x, torch.empty_like(x))

    c.attention_shared(0, batch, c.groups(sizes, shared), q, out)
    refused(batch, [2], [128])                       # not the whole batch
    refused(batch, [2, 2], [128, 64])
    refused(batch, [3, 0], [64, 0])
    refused(batch, [2, -1, 2], [64, 0, 0])
    refused(batch, [], [])
    refused(batch, [2, 1], [129, 64])                # past a request's first token
    refused(batch, [2, 1], [-1, 64])
    refused(batch, [1, 1, 1, 1], [0, 0, 0, 0])
    refused(c.batch([0, 1, 2], [130, 128, 64], [2, 2, 1]), sizes, shared, x=torch.zeros(5, 2, 128, dtype=BF, device="cuda"))  # more rows than room
    with pytest.raises(ValueError):
        c.groups([2, 1], [128])
    with pytest.raises(native.TssError):
        paged.Kv4Cache(c.pool, c.table, n_q_heads=2, n_kv_heads=2, head_dim=128, shared_rows=8193)
    c.attention_shared(0, c.batch([0, 1, 2], first, [0, 0, 0]), c.groups(sizes, shared), q[:0], out[:0])
    # a request without rows does not bound the shared tokens
    c.attention_shared(0, c.batch([0, 1, 2], [130, 5, 64], [2, 0, 1]), c.groups(sizes, shared), q[:3], out[:3])
    assert c.sync_status() == native.TSS_OK


def test_no_requests():
    """Refused, as by the other calls on a batch."""
    c, _, _ = shared_cache([1], [64], [64], [1], 2, 2, 128, seed=14)
    q = torch.zeros(0, 2, 128, dtype=BF, device="cuda")
    with pytest.raises(native.TssError):
        c.attention_shared(0, c.batch([], [], []), c.groups([], []), q, q.clone())
    assert c.sync_status() == native.TSS_OK
