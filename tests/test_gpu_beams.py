"""Beam selection against the definition in 64 bits: choices equal wherever the candidates are further apart than the values'
error, ties exactly by index, finished and dead beams, masked and bad rows, strides and types.

Tolerances.  A row's ln sum exp: terms carry 2^-22 of the fast exponential and 2^-24 a rounding in the exponent, the largest ones none
(64 bits); the sum of the others, of random sign, leaves 1e-7 at most.  The value is rounded once to fp32 (2^-24 of it)."""
import math

import pytest
import torch

from paper_2609_26100_gb300 import beams, native

pytestmark = pytest.mark.gpu
BF, HF, FL = torch.bfloat16, torch.float16, torch.float32


def definition(logits, score, n_beams, keep, done=None, end=0):
    """(value, parent, token) [groups][keep] in 64 bits; -inf, -1, -1 where a group offers less."""
    x = logits.double().cpu()
    x = torch.where(x <= -1e38, -math.inf, x)
    rows, vocab = x.shape
    s = torch.zeros(rows).double() if score is None else score.double().cpu()
    bad = torch.isnan(x).any(1) | (x >= 1e38).any(1) | ~torch.isfinite(s)
    top = x.amax(1, keepdim=True)
    lse = (top + (x - top).exp().sum(1, keepdim=True).log())
    v = torch.where(torch.isfinite(x) & ~bad[:, None], s[:, None] + (x - lse), -math.inf)
    if done is not None:
        for r in done.cpu().nonzero()[:, 0].tolist():
            v[r] = -math.inf
            if math.isfinite(s[r]):
                v[r, end] = s[r]
    v = torch.nan_to_num(v, nan=-math.inf, neginf=-math.inf)
    flat = v.view(rows // n_beams, -1)
    # (in a row the order is that of its logits, also where 64 bits of a value do not show their difference: the value is
    # score + x - lse, and x - y > 0 however small)
    order = torch.argsort(torch.nan_to_num(x, nan=-math.inf), dim=1, descending=True, stable=True) + torch.arange(rows)[:, None] * vocab
    order = order.view(rows // n_beams, -1) - torch.arange(rows // n_beams)[:, None] * (n_beams * vocab)
    best, at = torch.sort(flat.gather(1, order), dim=1, descending=True, stable=True)
    at = order.gather(1, at)
    k = min(keep, flat.shape[1])
    value = torch.full((flat.shape[0], keep), -math.inf, dtype=torch.float64)
    parent, token = torch.full((flat.shape[0], keep), -1), torch.full((flat.shape[0], keep), -1)
    value[:, :k] = best[:, :k]
    there = value > -math.inf
    base = torch.arange(flat.shape[0])[:, None] * n_beams
    parent[:, :k] = base + at[:, :k] // vocab
    token[:, :k] = at[:, :k] % vocab
    parent[~there] = token[~there] = -1
    return value, parent, token, v


def chosen(logits, score, n_beams, keep, done=None, end=0, selector=None):
    rows, vocab = logits.shape
    s = selector or beams.BeamSelector(rows, vocab, keep)
    g = rows // n_beams
    out = torch.full((g, keep), 5.0, device="cuda"), *(torch.full((g, keep), 77, dtype=torch.int32, device="cuda") for _ in range(2))
    s.select(logits, score, *out, n_beams=n_beams, done=done, end_token=end)
    return out, s


def compare(out, ref, n_beams):
    value, parent, token, v = ref
    got = [x.cpu() for x in out]
    there = value > -math.inf
    assert torch.equal(torch.isinf(got[0]), ~there)
    room = 1e-7 + value.abs() * 2.0 ** -24
    assert (torch.where(there, (got[0].double() - value).abs() - room, -1.0) <= 0).all(), float(torch.where(there, (got[0].double() - value).abs(), 0.0).max())
    same = (got[1] == parent) & (got[2] == token)
    # a place may differ only where another candidate's value lies within the error
    other = v[got[1].clamp(min=0).long(), got[2].clamp(min=0).long()]
    assert (same | (there & ((other - value).abs() <= 2e-7))).all()
    assert not (~same & ~there).any()
    pairs = (got[1].long() << 32 | got[2].long())
    for g in range(len(pairs)):
        mine = pairs[g][there[g]]
        assert len(mine.unique()) == len(mine)
    return same.all()


CASES = [  # rows, beams, vocab, keep, dtype
    (1, 1, 1, 1, FL), (1, 1, 1, 3, FL), (4, 4, 7, 5, BF), (6, 2, 33, 128, HF), (4, 4, 32000, 4, BF), (3, 3, 2047, 3, FL), (3, 3, 2048, 6, HF),
    (3, 1, 2049, 2, BF), (64, 64, 5001, 64, BF), (64, 8, 50021, 16, FL), (12, 4, 131072, 8, HF), (40, 5, 8193, 10, FL), (700, 7, 300, 14, BF),
    (2, 2, 400000, 128, BF), (64, 64, 40000, 128, FL), (320, 32, 20011, 32, BF),
]


@pytest.mark.parametrize("rows,n_beams,vocab,keep,dtype", CASES)
def test_definition(rows, n_beams, vocab, keep, dtype):
    g = torch.Generator(device="cuda").manual_seed(rows + vocab)
    x = torch.randn(rows, vocab, generator=g, device="cuda") * 2
    x.scatter_add_(1, torch.randint(vocab, (rows, 9), generator=g, device="cuda"), torch.full((rows, 9), 5.0, device="cuda"))
    score = torch.randn(rows, generator=g, device="cuda") - 9
    x = x.to(dtype)
    out, s = chosen(x, score, n_beams, keep)
    compare(out, definition(x, score, n_beams, keep), n_beams)
    again, _ = chosen(x, None, n_beams, keep, selector=s)
    compare(again, definition(x, None, n_beams, keep), n_beams)
    assert s.sync_status() == native.TSS_OK


@pytest.mark.parametrize("dtype", [BF, HF, FL])
@pytest.mark.parametrize("vocab,stride,offset", [(1000, 1000, 0), (1000, 1003, 1), (8195, 8195, 3), (50021, 50030, 0)])
def test_equal_rows_and_ties(dtype, vocab, stride, offset):
    """Equal rows, whatever their alignment, have equal values: ties go to the lowest beam, then the lowest token."""
    g = torch.Generator(device="cuda").manual_seed(3)
    row = (torch.randn(vocab, generator=g, device="cuda") * 2).to(dtype)
    row[torch.randint(vocab, (40,), generator=g, device="cuda")] = 6.0  # ties within a row too
    store = torch.zeros(8 * stride + offset, dtype=dtype, device="cuda")
    x = store[offset:offset + 8 * stride].view(8, stride)[:, :vocab]
    x[:] = row
    score = torch.full((8,), -3.25, device="cuda")
    out, s = chosen(x, score, 8, 20)
    value, parent, token, _ = definition(x, score, 8, 20)
    assert torch.equal(out[1].cpu().long(), parent) and torch.equal(out[2].cpu().long(), token)
    # all logits equal: the first tokens of the first beam
    store.fill_(1.5)
    out, _ = chosen(x, score, 4, 20, selector=s)
    assert out[1].tolist() == [[0] * 20, [4] * 20] and out[2].tolist() == [list(range(20))] * 2
    # zeros of either sign are equal
    store.zero_()
    store[offset + 5] = -0.0
    out, _ = chosen(x, score, 8, 8, selector=s)
    assert out[2].tolist() == [list(range(8))]


def test_sorted_and_flat_rows_with_many_kept():
    """Rows whose largest entries lie side by side, and rows all alike, at the most that can be kept."""
    vocab, rows, keep = 70000, 64, 128
    x = torch.arange(vocab, 0, -1, device="cuda").float().mul_(1e-3).repeat(rows, 1)
    out, s = chosen(x, None, 64, keep)
    value, parent, token, _ = definition(x, None, 64, keep)
    assert torch.equal(out[1].cpu().long(), parent) and torch.equal(out[2].cpu().long(), token)
    score = torch.full((rows,), -1e6, device="cuda")
    score[17] = 0.0  # one beam has all of them
    out, _ = chosen(x, score, 64, keep, selector=s)
    assert set(out[1].flatten().tolist()) == {17} and out[2].tolist() == [list(range(keep))]
    x.fill_(-2.0)
    out, _ = chosen(x, None, 64, keep, selector=s)
    assert set(out[1].flatten().tolist()) == {0} and out[2].tolist() == [list(range(keep))]


def test_finished_and_dead_beams():
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn(12, 3000, generator=g, device="cuda").to(BF)
    score = torch.tensor([-3.0, -2.0, -50.0, -math.inf, -math.inf, -math.inf, -1.0, -math.inf, -2.0, -7.0, -2.0, -9.0], device="cuda")
    done = torch.tensor([0, 1, 1, 0, 1, 0, 1, 0, 1, 1, 1, 1], dtype=torch.int32, device="cuda")
    out, s = chosen(x, score, 4, 6, done, 11)
    assert compare(out, definition(x, score, 4, 6, done, 11), 4)
    assert out[1][1].tolist() == [6, -1, -1, -1, -1, -1]         # one finished beam is all that the second group has
    assert out[1][2].tolist() == [8, 10, 9, 11, -1, -1]          # equal values: the lower beam
    assert out[2][2].tolist() == [11] * 4 + [-1] * 2
    # finished beams' logits are not read
    x[1:3] = math.nan
    again, _ = chosen(x, score, 4, 6, done, 11, selector=s)
    assert all(torch.equal(a, b) for a, b in zip(out, again)) and s.sync_status() == native.TSS_OK
    # a first step: one beam counts
    score = torch.tensor([0.0] + [-math.inf] * 3, device="cuda")
    first, s = chosen(x[5:9], score, 4, 4)
    assert compare(first, definition(x[5:9], score, 4, 4), 4) and set(first[1].flatten().tolist()) == {0}


def test_masked_and_bad_rows():
    g = torch.Generator(device="cuda").manual_seed(6)
    x = torch.randn(8, 9000, generator=g, device="cuda")
    x[0] = -math.inf                       # a row that offers nothing
    x[1, 5:] = torch.finfo(FL).min         # five tokens allowed
    x[2, :8000] = -math.inf
    x[3, 77] = -math.inf
    score = torch.randn(8, generator=g, device="cuda")
    out, s = chosen(x, score, 4, 40)
    assert compare(out, definition(x, score, 4, 40), 4) and s.sync_status() == native.TSS_OK
    y = x.clone()
    y[4, 8999] = math.nan
    y[5, 0] = math.inf
    y[6, 100] = 2e38
    out, _ = chosen(y, score, 4, 40, selector=s)
    assert compare(out, definition(y, score, 4, 40), 4) and s.sync_status() == native.TSS_ERR_DEVICE_CHECK
    assert set(out[1][1].tolist()) == {7}
    for odd in (math.nan, math.inf):
        z = score.clone()
        z[7] = odd
        out, _ = chosen(y, z, 4, 40, selector=s)
        assert s.sync_status() == native.TSS_ERR_DEVICE_CHECK
        assert out[1][1].tolist() == [-1] * 40 and torch.equal(out[2][1], out[1][1]) and torch.isinf(out[0][1]).all()
    # few tokens in all
    x[:] = -math.inf
    x[2, 100] = 1.0
    x[6, 8999] = x[7, 0] = -4e4
    out, _ = chosen(x, score, 4, 40, selector=s)
    assert compare(out, definition(x, score, 4, 40), 4) and s.sync_status() == native.TSS_OK


@pytest.mark.parametrize("size", [1e-30, 1.0, 3e4, 1e20, 9e37])
def test_magnitudes(size):
    g = torch.Generator(device="cuda").manual_seed(8)
    x = (torch.rand(6, 4000, generator=g, device="cuda") * 2 - 1) * size
    out, s = chosen(x, None, 3, 5)
    value, parent, token, v = definition(x, None, 3, 5)
    got = out[0].cpu().double()
    assert ((got - value).abs() <= 1e-7 + value.abs() * 2.0 ** -23).all()
    assert (out[1].cpu() == parent).all() and (out[2].cpu() == token).all()


def test_in_place_streams_and_graphs():
    g = torch.Generator(device="cuda").manual_seed(9)
    x = torch.randn(12, 32000, generator=g, device="cuda").to(BF)
    score = torch.randn(12, generator=g, device="cuda")
    ref, s = chosen(x, score, 4, 4)
    # score_out in score's place, on another stream, captured and replayed on other logits
    mine = score.clone()
    parent, token = (torch.zeros(3, 4, dtype=torch.int32, device="cuda") for _ in range(2))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        s.select(x, mine, mine.view(3, 4), parent, token, n_beams=4)
    side.synchronize()
    assert torch.equal(mine.view(3, 4), ref[0]) and torch.equal(parent, ref[1]) and torch.equal(token, ref[2])
    graph = torch.cuda.CUDAGraph()
    mine.copy_(score)
    y = x.clone()
    with torch.cuda.graph(graph):
        s.select(y, mine, mine.view(3, 4), parent, token, n_beams=4)
    for seed in range(3):
        y.copy_(torch.randn(12, 32000, generator=g, device="cuda"))
        was = mine.clone()
        graph.replay()
        want, _ = chosen(y, was, 4, 4)
        assert torch.equal(mine.view(3, 4), want[0]) and torch.equal(parent, want[1]) and torch.equal(token, want[2])


def test_refusals():
    x = torch.zeros(8, 100, device="cuda")
    s = beams.BeamSelector(8, 100, 4)
    i = lambda *shape: torch.zeros(*shape, dtype=torch.int32, device="cuda")  # noqa: E731
    f = lambda *shape: torch.zeros(*shape, device="cuda")  # noqa: E731
    score = f(8)

    def refused(*a, **kw):
        with pytest.raises((native.TssError, ValueError, TypeError)):
            s.select(*a, **{"n_beams": 4, **kw})

    refused(x, score, f(2, 5), i(2, 5), i(2, 5))                   # more kept than the workspace has room for
    refused(x, score, f(2, 0), i(2, 0), i(2, 0))
    refused(x, score, f(2, 4), i(2, 4), i(2, 4), n_beams=3)
    refused(x, score, f(2, 4), i(2, 4), i(2, 4), n_beams=0)
    refused(x, score[:7], f(2, 4), i(2, 4), i(2, 4))
    refused(x, score.double(), f(2, 4), i(2, 4), i(2, 4))
    refused(x, score, f(2, 4), i(2, 3), i(2, 4))
    refused(x, score, f(2, 4), i(2, 4), i(2, 4).long())
    refused(x, score, f(2, 4), i(2, 4).cpu(), i(2, 4))
    refused(x.cpu(), score, f(2, 4), i(2, 4), i(2, 4))
    refused(x[:, :99], score, f(2, 4), i(2, 4), i(2, 4))           # another vocabulary
    refused(x.t().contiguous().t(), score, f(2, 4), i(2, 4), i(2, 4))
    refused(x.int(), score, f(2, 4), i(2, 4), i(2, 4))
    refused(f(16, 100), f(16), f(4, 4), i(4, 4), i(4, 4))          # more rows
    refused(x, score, f(2, 4), i(2, 4), i(2, 4), done=i(8), end_token=100)
    refused(x, score, f(2, 4), i(2, 4), i(2, 4), done=i(8), end_token=-1)
    refused(x.expand(2, 8, 100).reshape(16, 100)[:8].as_strided((8, 100), (50, 1)), score, f(2, 4), i(2, 4), i(2, 4))
    s.select(x[:0], score[:0], f(0, 4), i(0, 4), i(0, 4), n_beams=4)
    for bad in ((0, 100, 4), (8, 0, 4), (8, 100, 0), (8, 100, 129), (8, 1 << 25, 4), (1 << 21, 100, 4)):
        with pytest.raises(native.TssError):
            beams.BeamSelector(*bad)
    assert s.sync_status() == native.TSS_OK


@pytest.mark.parametrize("rows,n_beams,vocab,keep,dtype", [(512, 32, 70001, 32, BF), (640, 16, 66000, 128, HF), (320, 8, 66001, 7, FL), (2048, 64, 9000, 64, BF)])
def test_many_long_rows(rows, n_beams, vocab, keep, dtype):
    """Chunks of up to sixteen tiles: random rows, flat ones, of which every element is as large as the bound, rising and falling ones.  The
    reference on the GPU, in 64 bits; candidates of equal value may come in either order where the logits are random."""
    g = torch.Generator(device="cuda").manual_seed(31)
    x = torch.randn(rows, vocab, generator=g, device="cuda").mul_(3).to(dtype)
    score = torch.randn(rows, generator=g, device="cuda")
    x[:n_beams] = 0.5
    score[:n_beams] = -1.0
    x[n_beams:2 * n_beams] = torch.linspace(-9, 9, vocab, device="cuda").to(dtype)
    x[2 * n_beams:3 * n_beams] = torch.linspace(9, -9, vocab, device="cuda").to(dtype)
    x[3 * n_beams + 1, vocab // 3:] = -math.inf
    (value, parent, token), s = chosen(x, score, n_beams, keep)
    assert s.sync_status() == native.TSS_OK
    for at in range(0, rows, n_beams):
        v = x[at:at + n_beams].double().log_softmax(-1) + score[at:at + n_beams].double()[:, None]
        top, i = v.reshape(-1).topk(keep), at // n_beams
        place = (parent[i].long() - at) * vocab + token[i].long()
        assert place.unique().numel() == keep and (place >= 0).all()
        # (a float's half step, and 1e-7 of the sum)
        assert ((value[i].double() - top.values).abs() <= top.values.abs() * 2.0 ** -24 + 2e-7).all()
        assert ((v.reshape(-1)[place] - top.values).abs() <= 2e-7).all()
    assert (parent[0] == 0).all() and torch.equal(token[0].long(), torch.arange(keep, device="cuda"))
