"""The paged 4-bit cache: appending, reading back and attention, against references in 64 bits.

Codes and parameters follow from correctly rounded fp32 operations, so appending is compared bit for bit.

Attention's tolerances.  Weights enter the product with the values as fp16 (2^-11 of the largest value
summed, at most), everything else is fp32; the output is rounded once (2^-8 of its magnitude covers half an
ulp of bf16, 2^-11 of fp16).  The scores' fp32 sums of 128 products and the sum of the weights leave
lse within 2e-5 of the largest score's magnitude and one."""
import math
import random

import pytest
import torch

import paged_ref as R
from paper_2609_26100_gb300 import native, paged

pytestmark = pytest.mark.gpu


def make(lens, hq, hk, d, seed=0, layers=1, spare=2, poison=True):
    """A cache whose pages lie in random order; what no append has written is NaN parameters."""
    need = [max(1, -(-n // 64)) for n in lens]
    g = torch.Generator().manual_seed(seed)
    ids = torch.randperm(sum(need) + spare, generator=g).tolist()
    table = torch.full((len(lens), max(need)), -1, dtype=torch.int32)
    at = 0
    for b, m in enumerate(need):
        table[b, :m] = torch.tensor(ids[at:at + m], dtype=torch.int32)
        at += m
    pool = torch.full((layers, sum(need) + spare, paged.page_bytes(hk, d)), 0xFF if poison else 0, dtype=torch.uint8, device="cuda")
    return paged.Kv4Cache(pool, table.cuda(), n_q_heads=hq, n_kv_heads=hk, head_dim=d)


def fill(cache, lens, seed=0, dtype=torch.bfloat16, layer=0, scale=1.0):
    """Append whole sequences; returns (k, v) as they are stored, in 64 bits, [seq] -> [n][hk][d]."""
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    n, hk, d = sum(lens), cache.n_kv_heads, cache.head_dim
    k = (torch.randn(n, hk, d, generator=g, device="cuda") * scale).to(dtype)
    v = (torch.randn(n, hk, d, generator=g, device="cuda") * scale).to(dtype)
    cache.append(layer, cache.batch(list(range(len(lens))), [0] * len(lens), lens), k, v)
    return [list(R.stored(x).split(list(lens))) for x in (k, v)]


def close(out, lse, ref, ref_lse, vmax, smax):
    bound = ref.abs() * 2.0 ** -8 + vmax * 2.0 ** -10
    assert ((out.double() - ref).abs() <= bound).all(), float(((out.double() - ref).abs() - bound).max())
    inf = torch.isinf(ref_lse)
    assert torch.equal(inf, torch.isinf(lse))
    assert (torch.where(inf, 0.0, lse.double() - ref_lse).abs() <= 2e-5 * (1 + smax)).all()


# ------------------------------------------------------------------------------------------------
# append and read
# ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("first,n", [((0,), (1,)), ((0, 5, 64), (64, 3, 128)), ((63, 31, 40, 7), (2, 1, 0, 121)), ((95,), (33,))])
def test_append_and_read(d, dtype, first, n):
    hk = 3
    lens = [f + m for f, m in zip(first, n)]
    cache = make(lens, hk, hk, d)
    old = fill(cache, list(first), dtype=dtype)
    before = cache.pool.clone()
    g = torch.Generator(device="cuda").manual_seed(7)
    fused = (torch.randn(sum(n), 2 * hk, d, generator=g, device="cuda") * torch.rand(sum(n), 2 * hk, 1, generator=g, device="cuda") * 5).to(dtype)
    k, v = fused[:, :hk], fused[:, hk:]
    cache.append(0, cache.batch(list(range(len(n))), first, n), k, v)
    for side, x in enumerate((k, v)):
        at = 0
        for b, m in enumerate(n):
            want = torch.cat([old[side][b], R.stored(x[at:at + m])])
            assert torch.equal(R.sequence_values(cache.pool[0], cache.table, b, lens[b], hk, d, side), want)
            at += m
    # tokens that the call did not bring keep their nibbles and parameters
    pos = {int(cache.table[b, t // 64]) * 64 + t % 64 for b, (f, m) in enumerate(zip(first, n)) for t in range(f, f + m)}
    tok = torch.tensor([i not in pos for i in range(cache.pool.shape[1] * 64)], device="cuda").view(-1, 1, 64)
    for side in (0, 1):
        was, now = (p[0].view(p.shape[1], hk, -1) for p in (before, cache.pool))
        assert ((R.codes_of(was, d, side) == R.codes_of(now, d, side)).all(-1) | ~tok).all()
        assert ((R.params_of(was, d, side).view(torch.int16) == R.params_of(now, d, side).view(torch.int16)).flatten(-2).all(-1) | ~tok).all()
    # and back
    batch = cache.batch(list(range(len(n))), [0] * len(n), lens)
    ko, vo = (torch.empty(sum(lens), hk, d, dtype=torch.float32, device="cuda") for _ in range(2))
    cache.read(0, batch, ko, vo)
    for side, o in enumerate((ko, vo)):
        want = torch.cat([R.sequence_values(cache.pool[0], cache.table, b, m, hk, d, side) for b, m in enumerate(lens)])
        assert torch.equal(o, want.float())
    one = torch.empty(sum(lens), hk, d, dtype=dtype, device="cuda")
    cache.read(0, batch, None, one)
    assert torch.equal(one, vo.to(dtype))
    assert cache.sync_status() == native.TSS_OK


def test_extreme_values():
    """Constant groups, values past fp16's range, tiny ones, NaN and infinities."""
    cache = make([64], 1, 1, 128)
    x = torch.randn(64, 1, 128, device="cuda")
    x[0] = 3.0
    x[1, :, :64] = 1e30
    x[2, :, 5] = -2e6
    x[3] *= 1e-7
    x[4, :, 70] = math.nan
    x[5, :, 0] = math.inf
    x[6] = 0.0
    x[7] = 1e-30
    x[8, :, 3] = -math.inf
    cache.append(0, cache.batch([0], [0], [64]), x, x)
    want = R.stored(x)
    for side in (0, 1):
        got = R.sequence_values(cache.pool[0], cache.table, 0, 64, 1, 128, side)
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))
    assert torch.isnan(want[4, 0, 64:]).all() and not torch.isnan(want[4, 0, :64]).any()
    # the error of an ordinary group: half a step of its range / 15, and the rounding of s and z to fp16
    y, g = want[10:], x[10:].double()
    for lo in (0, 64):
        span = g[..., lo:lo + 64].amax(-1) - g[..., lo:lo + 64].amin(-1)
        assert ((y - g)[..., lo:lo + 64].abs().amax(-1) <= span / 30 + span * 2.0 ** -10 + 2.0 ** -9).all()


def test_layers_and_wrong_pages():
    cache = make([100, 64], 2, 2, 64, layers=3)
    k = torch.randn(164, 2, 64, device="cuda")
    cache.append(1, cache.batch([0, 1], [0, 0], [100, 64]), k, k)
    assert (cache.pool[0] == 0xFF).all() and (cache.pool[2] == 0xFF).all()
    cache.table[0, 1] = cache.pool.shape[1]  # past the pool
    before = cache.pool.clone()
    cache.append(0, cache.batch([0], [64], [36]), k[64:100], k[64:100])
    assert torch.equal(cache.pool, before)
    assert cache.sync_status() == native.TSS_ERR_DEVICE_CHECK
    assert cache.sync_status() == native.TSS_OK
    out = torch.full((100, 2, 64), 7.0, device="cuda")
    cache.read(1, cache.batch([0], [0], [100]), out, None)
    assert (out[64:] == 0).all() and not (out[:64] == 0).all()
    assert cache.sync_status() == native.TSS_ERR_DEVICE_CHECK
    q = torch.randn(1, 2, 64, device="cuda", dtype=torch.bfloat16)
    cache.attention(1, cache.batch([0], [99], [1]), q, q.clone())
    assert cache.sync_status() == native.TSS_ERR_DEVICE_CHECK
    cache.table[0, 1] = -1
    cache.attention(1, cache.batch([0], [99], [1]), q, q.clone())
    assert cache.sync_status() == native.TSS_ERR_DEVICE_CHECK


# ------------------------------------------------------------------------------------------------
# attention
# ------------------------------------------------------------------------------------------------
def random_sets(n, rng):
    """Random ancestor-or-self sets of a tree, and depths."""
    sets, depth = [], []
    for i in range(n):
        p = -1 if i == 0 else rng.randrange(max(0, i - 5), i)
        sets.append((sets[p] if p >= 0 else 0) | 1 << i)
        depth.append(depth[p] + 1 if p >= 0 else 0)
    return sets, depth


def run_attention(first, n, hq, hk, d, dtype, window=0, sinks=0, tree=False, seed=0, sets=None, qscale=2.0, scale=None, spread=False):
    rng = random.Random(seed)
    lens = [f + m for f, m in zip(first, n)]
    cache = make(lens, hq, hk, d, seed=seed)
    k, v = fill(cache, lens, seed=seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 5)
    rows = sum(n)
    q = (torch.randn(rows, hq + 1, d, generator=g, device="cuda") * qscale).to(dtype)[:, :hq]  # a slice of wider rows
    wide = torch.full((rows, hq + 2, d), 3.0, dtype=dtype, device="cuda")
    out, lse = wide[:, :hq], torch.empty(rows, hq, device="cuda")
    trees = [random_sets(m, rng) for m in n]
    if sets is None:
        sets = [t[0] if tree else None for t in trees]
    pos = [[f + x for x in (t[1] if tree else range(m))] for f, m, t in zip(first, n, trees)]
    flat = [w for s in sets if s is not None for w in R.words(s)]
    mask = torch.tensor(flat, dtype=torch.int64, device="cuda").view(-1, 2) if flat else None
    positions = torch.tensor([p for x in pos for p in x], dtype=torch.int32, device="cuda") if tree else None
    cache.attention(0, cache.batch(list(range(len(n))), first, n), q, out, lse=lse, window=window, sinks=sinks, mask=mask,
                    positions=positions, scale=scale)
    assert cache.sync_status() == native.TSS_OK
    assert (wide[:, hq:] == 3.0).all()
    at = 0
    s = d ** -0.5 if scale is None else scale
    for b, m in enumerate(n):
        see = R.sees(first[b], m, sets[b], pos[b], window, sinks, "cuda")
        ref, ref_lse = R.attention(k[b], v[b], q[at:at + m].double(), see, s)
        smax = float((q[at:at + m].double().norm(dim=-1).amax() if m else 0) * (k[b].norm(dim=-1).amax() if len(k[b]) else 0) * s)
        close(out[at:at + m], lse[at:at + m], ref, ref_lse, float(v[b].abs().amax()) if len(v[b]) else 0.0, smax)
        at += m
    return cache


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hk", [(2, 2), (6, 2), (8, 1)])
@pytest.mark.parametrize("first,n", [((0,), (1,)), ((64,), (1,)), ((63,), (1,)), ((62, 0, 130), (6, 5, 0)), ((300, 17, 1), (9, 1, 33)),
                                     ((1000, 3), (1, 70)), ((40,), (128,))])
def test_chains(dtype, d, hq, hk, first, n):
    run_attention(first, n, hq, hk, d, dtype)


@pytest.mark.parametrize("d,hq,hk", [(128, 4, 4), (128, 8, 2), (64, 4, 1)])
@pytest.mark.parametrize("first,n", [((70,), (61,)), ((0, 200, 511), (128, 7, 65)), ((129,), (2,))])
def test_trees(d, hq, hk, first, n):
    run_attention(first, n, hq, hk, d, torch.bfloat16, tree=True, seed=3)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 0), (64, 4), (65, 0), (100, 64), (100, 65), (128, 1000), (5000, 3), (200, 130)])
@pytest.mark.parametrize("tree", [False, True])
def test_windows_and_sinks(window, sinks, tree):
    run_attention((500, 64, 0, 129, 700), (3, 9, 20, 1, 40), 4, 2, 128, torch.bfloat16, window=window, sinks=sinks, tree=tree, seed=2)
    run_attention((333, 640), (1, 66), 2, 2, 64, torch.float16, window=window, sinks=sinks, tree=tree, seed=4)


def test_rows_that_see_nothing():
    """Masks that leave a row no key: zeros and -infinity, and the other rows are not touched by it."""
    sets = [[0, 1, 0, 0b1010], [0b1, 0, 0b111]]
    run_attention((0, 0), (4, 3), 4, 2, 128, torch.bfloat16, sets=sets)
    run_attention((0, 0), (4, 3), 4, 4, 64, torch.bfloat16, sets=sets)
    many = [[0 if i % 3 else 1 << (i // 2) for i in range(100)]]
    run_attention((0,), (100,), 2, 2, 128, torch.bfloat16, sets=many)


@pytest.mark.parametrize("scale,qscale", [(1.0, 8.0), (1e-3, 1.0), (0.5, 60.0), (1.0, 1e-6)])
def test_steep_and_flat_scores(scale, qscale):
    """One key takes all the weight, or all share it; queries of any magnitude."""
    run_attention((777, 100), (5, 40), 4, 2, 128, torch.bfloat16, scale=scale, qscale=qscale)


def test_values_of_any_magnitude():
    """V scales from fp16's smallest to large ones side by side, and tokens whose values are all equal."""
    cache = make([200], 2, 2, 128)
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn(200, 2, 128, generator=g, device="cuda") for _ in range(2))
    v *= 10.0 ** torch.linspace(-9, 4, 200, device="cuda")[torch.randperm(200, generator=g, device="cuda")][:, None, None]
    v[50:60] = 0.0
    v[70] = 5.0
    cache.append(0, cache.batch([0], [0], [200]), k, v)
    q = (torch.randn(6, 2, 128, generator=g, device="cuda") * 6).bfloat16()
    out, lse = torch.empty_like(q), torch.empty(6, 2, device="cuda")
    cache.attention(0, cache.batch([0], [194], [6]), q, out, lse=lse)
    see = R.sees(194, 6, None, range(194, 200), 0, 0, "cuda")
    sk, sv = R.stored(k), R.stored(v)
    ref, ref_lse = R.attention(sk, sv, q.double(), see, 128 ** -0.5)
    # each weight is off by 2^-11 of itself at most, so an output by 2^-11 of the weighted magnitudes
    mag = torch.zeros_like(ref)
    for i in range(6):
        for h in range(2):
            w = torch.softmax(torch.where(see[i], sk[:, h] @ q[i, h].double() * 128 ** -0.5, -math.inf), 0)
            mag[i, h] = w @ sv[:, h].abs()
    assert ((out.double() - ref).abs() <= ref.abs() * 2.0 ** -8 + mag * 2.0 ** -9).all()
    assert ((lse.double() - ref_lse).abs() <= 2e-4).all()
    only = torch.empty(1, 2, 128, dtype=torch.bfloat16, device="cuda")
    cache.attention(0, cache.batch([0], [0], [1]), q[:1], only)
    assert ((only[0].double() - sv[0]).abs() <= sv[0].abs() * 2.0 ** -8 + 1e-12).all()


@pytest.mark.parametrize("rows", [1, 6, 40])
@pytest.mark.parametrize("d", [64, 128])
def test_what_no_row_sees_does_not_reach_it(rows, d):
    """NaN in keys and values past the block, outside the window and in block rows that the mask hides."""
    first = 300
    cache = make([first + rows + 20], 4, 2, d)
    k, v = fill(cache, [first + rows], seed=9)
    bad = torch.full((1, 2, d), math.nan, device="cuda")
    q = torch.randn(rows, 4, d, device="cuda", dtype=torch.bfloat16)
    for t in list(range(10, 100)) + [first + rows + 3]:
        cache.append(0, cache.batch([0], [t], [1]), bad, bad)
    sets = [1 << i for i in range(rows)]
    if rows > 2:  # nobody sees row 1 of the block
        sets[1] = 1
        cache.append(0, cache.batch([0], [first + 1], [1]), bad, bad)
    mask = torch.tensor(R.words(sets), dtype=torch.int64, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(rows, 4, device="cuda")
    cache.attention(0, cache.batch([0], [first], [rows]), q, out, lse=lse, window=150, sinks=9, mask=mask)
    see = R.sees(first, rows, sets, range(first, first + rows), 150, 9, "cuda")
    ref, ref_lse = R.attention(k[0], v[0], q.double(), see, d ** -0.5)
    close(out, lse, ref, ref_lse, float(v[0].abs().amax()), 40.0)
    # and a NaN that is seen does reach the rows that see it
    cache.attention(0, cache.batch([0], [first], [rows]), q, out, lse=lse)
    assert torch.isnan(out).all() and torch.isnan(lse).all()


def test_shared_pages_and_many_requests():
    """64 requests over shared pages, the same sequence more than once."""
    cache = make([200, 65], 4, 4, 128)
    k, v = fill(cache, [200, 65], seed=11)
    seqs = [i % 2 for i in range(64)]
    first = [(190 if s == 0 else 60) - i // 8 for i, s in enumerate(seqs)]
    n = [1 + i % 3 for i in range(64)]
    q = torch.randn(sum(n), 4, 128, device="cuda", dtype=torch.float16)
    out, lse = torch.empty_like(q), torch.empty(sum(n), 4, device="cuda")
    cache.attention(0, cache.batch(seqs, first, n), q, out, lse=lse)
    at = 0
    for s, f, m in zip(seqs, first, n):
        see = R.sees(f, m, None, range(f, f + m), 0, 0, "cuda")
        ref, ref_lse = R.attention(k[s][:f + m], v[s][:f + m], q[at:at + m].double(), see, 128 ** -0.5)
        close(out[at:at + m], lse[at:at + m], ref, ref_lse, 5.0, 40.0)
        at += m


@pytest.mark.parametrize("n", [1, 9, 61])
def test_long_context(n):
    """Many keys: the work of one (request, head) is shared, twice with the same bits."""
    first, hq, hk = 20011, 4, 2
    cache = make([first + n], hq, hk, 128)
    k, v = fill(cache, [first + n], seed=13)
    q = torch.randn(n, hq, 128, device="cuda", dtype=torch.bfloat16) * 3
    outs = []
    for _ in range(2):
        out, lse = torch.empty_like(q), torch.empty(n, hq, device="cuda")
        cache.attention(0, cache.batch([0], [first], [n]), q, out, lse=lse)
        outs.append((out, lse))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
    see = R.sees(first, n, None, range(first, first + n), 0, 0, "cuda")
    ref, ref_lse = R.attention(k[0], v[0], q.double(), see, 128 ** -0.5)
    close(out, lse, ref, ref_lse, 5.0, 60.0)


def test_pages_far_into_a_large_pool():
    """Byte offsets past 2^32."""
    n = (1 << 32) // paged.page_bytes(8, 128) + 40
    pool = torch.zeros(1, n, paged.page_bytes(8, 128), dtype=torch.uint8, device="cuda")
    table = torch.tensor([[n - 1, 0, n - 7]], dtype=torch.int32, device="cuda")
    cache = paged.Kv4Cache(pool, table, n_q_heads=8, n_kv_heads=8, head_dim=128)
    k, v = fill(cache, [150])
    q = torch.randn(2, 8, 128, device="cuda", dtype=torch.bfloat16)
    out, lse = torch.empty_like(q), torch.empty(2, 8, device="cuda")
    cache.attention(0, cache.batch([0], [148], [2]), q, out, lse=lse)
    see = R.sees(148, 2, None, (148, 149), 0, 0, "cuda")
    ref, ref_lse = R.attention(k[0], v[0], q.double(), see, 128 ** -0.5)
    close(out, lse, ref, ref_lse, 5.0, 40.0)


def test_another_stream():
    cache = make([300], 4, 4, 128)
    fill(cache, [300])
    q = torch.randn(6, 4, 128, device="cuda", dtype=torch.bfloat16)
    want, got = torch.empty_like(q), torch.empty_like(q)
    batch = cache.batch([0], [294], [6])
    cache.attention(0, batch, q, want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        cache.attention(0, batch, q, got)
    torch.cuda.synchronize()
    assert torch.equal(want, got)


# ------------------------------------------------------------------------------------------------
# refusals
# ------------------------------------------------------------------------------------------------
def test_refusals():
    cache = make([200, 64], 4, 2, 128)
    k = torch.zeros(4, 2, 128, device="cuda", dtype=torch.bfloat16)
    q = torch.zeros(4, 4, 128, device="cuda", dtype=torch.bfloat16)

    def status(call, *a, **kw):
        with pytest.raises(native.TssError) as e:
            call(*a, **kw)
        return e.value.status

    bad = native.TSS_ERR_INVALID_ARG
    B = cache.batch
    assert status(cache.append, 1, B([0], [0], [4]), k, k) == bad
    assert status(cache.append, -1, B([0], [0], [4]), k, k) == bad
    assert status(cache.append, 0, B([2], [0], [4]), k, k) == bad
    assert status(cache.append, 0, B([0], [-1], [4]), k, k) == bad
    assert status(cache.append, 0, B([0, 0], [0, 2], [2, 2]), k, k) == bad
    assert status(cache.append, 0, B([0], [253], [4]), k, k) == native.TSS_ERR_KV_CAPACITY
    assert status(cache.attention, 0, B([0], [253], [4]), q, q.clone()) == native.TSS_ERR_KV_CAPACITY
    assert status(cache.read, 0, B([0], [253], [4]), k, k) == native.TSS_ERR_KV_CAPACITY
    for kw in ({"scale": 0.0}, {"scale": math.nan}, {"scale": math.inf}, {"window": -1}, {"sinks": -1}):
        assert status(cache.attention, 0, B([0], [0], [4]), q, q.clone(), **kw) == bad
    long = torch.zeros(129, 4, 128, device="cuda", dtype=torch.bfloat16)
    assert status(cache.attention, 0, B([0], [0], [129]), long, long.clone()) == bad
    single = torch.zeros(4, 4, 128, device="cuda")
    assert status(cache.attention, 0, B([0], [0], [4]), single, single.clone()) == bad  # (fp32 queries)
    assert status(cache.attention, 0, B([0] * 65, [0] * 65, [0] * 64 + [4]), q, q.clone()) == bad
    odd = torch.zeros(4 * 4 * 128 + 1, device="cuda", dtype=torch.bfloat16)[1:].view(4, 4, 128)
    assert status(cache.attention, 0, B([0], [0], [4]), odd, q.clone()) == bad
    assert status(cache.attention, 0, B([0], [0], [4]), q, odd) == bad
    odd = torch.zeros(4 * 2 * 128 + 1, device="cuda", dtype=torch.bfloat16)[1:].view(4, 2, 128)
    assert status(cache.append, 0, B([0], [0], [4]), odd, k) == bad
    assert status(cache.read, 0, B([0], [0], [4]), k, odd) == bad
    with pytest.raises(ValueError):
        cache.append(0, B([0], [0], [5]), k, k)
    with pytest.raises(ValueError):
        cache.attention(0, B([0], [0], [4]), q.transpose(0, 1), q.clone())
    with pytest.raises(TypeError):
        cache.append(0, B([0], [0], [4]), k.double(), k.double())
    # nothing above left work or an error behind; empty calls are fine
    cache.append(0, B([0], [0], [0]), k[:0], k[:0])
    cache.attention(0, B([0, 1], [5, 0], [0, 0]), q[:0], q[:0].clone())
    assert (cache.pool == 0xFF).all() and cache.sync_status() == native.TSS_OK


@pytest.mark.parametrize("shape", [(4, 0, 128), (4, 3, 128), (0, 1, 128), (4, 4, 96), (130, 2, 64), (2048, 1025, 64)])
def test_create_refusals(shape):
    import ctypes
    h = ctypes.c_void_p()
    assert native.lib().tss_paged_create(*shape, ctypes.byref(h)) == native.TSS_ERR_INVALID_ARG and not h.value


def test_many_workspaces():
    """Handles that are made and dropped leave the memory as it was."""
    torch.cuda.synchronize()
    import ctypes
    free = []
    for i in range(3):
        for _ in range(20):
            h = ctypes.c_void_p()
            assert native.lib().tss_paged_create(32, 8, 128, ctypes.byref(h)) == native.TSS_OK
            native.lib().tss_paged_destroy(h)
        free.append(torch.cuda.mem_get_info()[0])
    assert free[1] == free[2]
