"""Appending with the norms and the rotation on the way: the bits of the two calls that it stands for, the definition in 64
bits, and its refusals."""
import math

import pytest
import torch

import paged_ref as R
from paper_2609_26100_gb300 import native, paged
from test_gpu_paged import make

pytestmark = pytest.mark.gpu
BF, HF, FL = torch.bfloat16, torch.float16, torch.float32


def table_of(rot, positions):
    freq, factor = native.rope_frequencies(rot, 10000.0, "yarn", 4.0, 512.0)
    t = torch.empty(positions, rot // 2, 2, device="cuda")
    native.rope_table(freq, t, factor)
    return t


def rows_of(n, hq, hk, d, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    fused = torch.randn(n, hq + 2 * hk, d, generator=g, device="cuda")
    fused[:, :, ::17] *= 3.0
    fused = fused.to(dtype)
    return fused[:, :hq], fused[:, hq:hq + hk], fused[:, hq + hk:]


def gains(d, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed + 99)
    return [(1 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(dtype) for _ in range(2)]


CASES = [  # d, dtype, rot, interleaved, norm, hq, hk, first, n
    (128, BF, 128, False, True, 8, 2, (0,), (1,)),
    (128, BF, 128, True, False, 4, 4, (0, 5, 64), (64, 3, 130)),
    (128, HF, 64, False, True, 6, 3, (63, 31, 40, 7), (2, 1, 0, 121)),
    (128, FL, 96, False, True, 2, 1, (95,), (33,)),
    (128, FL, 128, True, True, 3, 3, (1, 200), (31, 77)),
    (64, BF, 64, False, True, 5, 5, (17, 0), (50, 200)),
    (64, HF, 32, True, False, 4, 1, (30,), (5,)),
    (64, FL, 48, False, False, 1, 1, (0, 33), (65, 1)),
    (128, BF, 0, False, True, 4, 2, (10,), (40,)),
    (128, BF, 0, False, False, 0, 2, (10,), (40,)),
    (64, BF, 64, False, True, 0, 3, (0, 9), (3, 64)),
]


@pytest.mark.parametrize("d,dtype,rot,inter,norm,hq,hk,first,n", CASES)
@pytest.mark.parametrize("keep_k", [False, True])
def test_bits_of_the_two_calls(d, dtype, rot, inter, norm, hq, hk, first, n, keep_k):
    lens, rows = [f + m for f, m in zip(first, n)], sum(n)
    one, two = (make(lens, max(hq, hk) // hk * hk or hk, hk, d) for _ in range(2))
    q, k, v = rows_of(rows, hq, hk, d, dtype, 3)
    qg, kg = gains(d, dtype, 3) if norm else (None, None)
    t = table_of(rot, 1000) if rot else None
    # (positions other than the tokens' places, as of a tree)
    pos = torch.cat([torch.arange(f, f + m, device="cuda") // 2 for f, m in zip(first, n)]).to(torch.int32)
    kw = dict(q_gain=qg if hq else None, k_gain=kg, interleaved=inter)
    qo, ko = [torch.full_like(x, 7.0).contiguous() for x in (q, k)], None
    qo2, ko2 = (torch.empty(x.shape, dtype=dtype, device="cuda") for x in (q, k))
    ko = torch.empty(k.shape, dtype=dtype, device="cuda") if keep_k else None
    a = native.rope_args(q if hq else None, k, qo[0] if hq else None, ko, pos, t, to_pages=True, **kw)
    batch = one.batch(list(range(len(n))), first, n)
    one.append_rope(0, batch, a, v)
    native.qk_rope(native.rope_args(q if hq else None, k, qo2 if hq else None, ko2, pos, t, **kw))
    two.append(0, two.batch(list(range(len(n))), first, n), ko2, v)
    assert one.sync_status() == native.TSS_OK
    assert torch.equal(one.pool, two.pool)
    if hq:
        assert torch.equal(qo[0], qo2)
    if keep_k:
        assert torch.equal(ko, ko2)


@pytest.mark.parametrize("d,dtype,rot,inter,norm,hq,hk,first,n", CASES[:8])
def test_definition(d, dtype, rot, inter, norm, hq, hk, first, n):
    """Against 64 bits.  Rotated values: fp32 operations (the norm's and the rotation's, 16 roundings of 2^-24 of the pair's
    magnitude at most) and the type's half step.  Held values: half a code, and the roundings of s and z to fp16 (2^-11 of
    15 s and of z)."""
    lens, rows = [f + m for f, m in zip(first, n)], sum(n)
    cache = make(lens, hq // hk * hk or hk, hk, d)
    q, k, v = rows_of(rows, hq, hk, d, dtype, 5)
    qg, kg = gains(d, dtype, 5) if norm else (None, None)
    t = table_of(rot, 1000)
    pos = torch.cat([torch.arange(f, f + m, device="cuda") for f, m in zip(first, n)]).to(torch.int32)
    qo = torch.empty(q.shape, dtype=dtype, device="cuda")
    batch = cache.batch(list(range(len(n))), first, n)
    cache.append_rope(0, batch, native.rope_args(q, k, qo, None, pos, t, q_gain=qg, k_gain=kg, eps=1e-5, interleaved=inter, to_pages=True), v)
    back = [torch.empty(rows, hk, d, device="cuda") for _ in range(2)]
    cache.read(0, batch, *back)
    i = torch.arange(rot // 2, device="cuda")
    a, b = (2 * i, 2 * i + 1) if inter else (i, i + rot // 2)
    cs = t.double()[pos.long()][:, None]
    half = torch.finfo(dtype).eps / 2

    def rotated(x, gain):
        y = x.double()
        if gain is not None:
            y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-5) * gain.double()
        z, size = y.clone(), y.abs()
        z[..., a] = y[..., a] * cs[..., 0] - y[..., b] * cs[..., 1]
        z[..., b] = y[..., b] * cs[..., 0] + y[..., a] * cs[..., 1]
        size[..., a] = size[..., b] = (y[..., a].abs() + y[..., b].abs()) * cs.abs().amax()
        return z, z.abs() * half + size * 16 * 2.0 ** -24

    want, off = rotated(q, qg)
    assert ((qo.double() - want).abs() <= off).all()
    for got, (want, off) in zip(back, (rotated(k, kg), (v.double(), torch.zeros_like(v, dtype=torch.float64)))):
        span = want.unflatten(-1, (-1, 64))
        s, z = (span.amax(-1) - span.amin(-1)) / 15, span.amin(-1).abs()
        room = (s / 2 + 2 * (15 * s + z) * 2.0 ** -11 + 1e-6)[..., None].expand(span.shape).flatten(-2) + 3 * off.amax(-1, keepdim=True)
        assert ((got.double() - want).abs() <= room).all()


def test_positions_outside_the_table_and_missing_pages():
    cache = make([70, 10], 4, 2, 128)
    q, k, v = rows_of(80, 4, 2, 128, BF, 8)
    t = table_of(128, 32)
    pos = torch.arange(80, dtype=torch.int32, device="cuda")  # 32 .. 79 lie outside: as position 31
    pos[3] = -4
    qo, qr = torch.empty(80, 4, 128, dtype=BF, device="cuda"), torch.empty(80, 4, 128, dtype=BF, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    batch = cache.batch([0, 1], [0, 0], [70, 10])
    cache.append_rope(0, batch, native.rope_args(q, k, qo, None, pos, t, to_pages=True, status=status), v)
    assert int(status) == native.TSS_ERR_DEVICE_CHECK and cache.sync_status() == native.TSS_OK
    native.qk_rope(native.rope_args(q, None, qr, None, pos.clamp(0, 31), t))
    assert torch.equal(qo, qr)
    cache.append_rope(0, batch, native.rope_args(q, k, qo, None, pos, t, to_pages=True), v)
    assert cache.sync_status() == native.TSS_ERR_DEVICE_CHECK
    # sequence 0 without its second page: the other tokens are as before, q is whole
    cache.table[0, 1] = -1
    before = cache.pool.clone()
    ko = torch.empty(80, 2, 128, dtype=BF, device="cuda")
    qo.zero_()
    cache.append_rope(0, batch, native.rope_args(q, k, qo, ko, pos.clamp(0, 31), t, to_pages=True), v)
    assert cache.sync_status() == native.TSS_ERR_DEVICE_CHECK and cache.sync_status() == native.TSS_OK
    assert torch.equal(cache.pool, before) and torch.equal(qo, qr) and torch.isfinite(ko.float()).all()


def test_in_place_on_a_stream_and_in_a_graph():
    lens = [100, 37]
    one, two = make(lens, 4, 4, 64), make(lens, 4, 4, 64)
    q, k, v = rows_of(137, 4, 4, 64, BF, 9)
    t, pos = table_of(64, 200), torch.arange(137, dtype=torch.int32, device="cuda")
    q2, k2 = q.clone(), k.clone()
    ref = native.rope_args(q2, k2, q2, k2, pos, t)
    native.qk_rope(ref)
    batch = one.batch([0, 1], [0, 0], lens)
    two.append(0, batch, k2, v)
    qi, ki = q.clone(), k.clone()
    args = native.rope_args(qi, ki, qi, ki, pos, t, to_pages=True)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        one.append_rope(0, batch, args, v)
    side.synchronize()
    assert torch.equal(one.pool, two.pool) and torch.equal(qi, q2) and torch.equal(ki, k2)
    # captured, and replayed on other rows
    qo = torch.empty_like(qi)
    args = native.rope_args(qi, ki, qo, None, pos, t, to_pages=True)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one.append_rope(0, batch, args, v)
    qi.copy_(q.flip(0)), ki.copy_(k.flip(0))
    graph.replay()
    torch.cuda.synchronize()
    q2.copy_(q.flip(0)), k2.copy_(k.flip(0))
    native.qk_rope(ref)
    two.append(0, batch, k2, v)
    assert torch.equal(one.pool, two.pool) and torch.equal(qo, q2)


def test_refusals():
    cache = make([64], 4, 2, 128)
    q, k, v = rows_of(8, 4, 2, 128, BF, 1)
    t, pos = table_of(128, 64), torch.arange(8, dtype=torch.int32, device="cuda")
    qo = torch.empty(8, 4, 128, dtype=BF, device="cuda")
    batch = cache.batch([0], [0], [8])
    args = lambda **kw: native.rope_args(q, k, qo, None, pos, t, to_pages=True, **kw)  # noqa: E731
    before = cache.pool.clone()

    def refused(b, a, x):
        with pytest.raises((native.TssError, ValueError, TypeError)):
            cache.append_rope(0, b, a, x)

    refused(cache.batch([0], [0], [7]), args(), v[:7])               # other rows than the batch's
    refused(cache.batch([0, 0], [0, 4], [4, 4]), args(), v)          # a sequence twice
    refused(batch, args(), v.half())                                 # another type
    refused(batch, args(), v[:, :1])                                 # other heads
    refused(batch, native.rope_args(q, q, qo, None, pos, t, to_pages=True), v)   # keys of other heads
    refused(batch, native.rope_args(q, None, qo, None, pos, t, to_pages=True), v)
    refused(batch, args(eps=-1.0, k_gain=torch.ones(128, dtype=BF, device="cuda")), v)
    refused(batch, args(eps=math.nan, k_gain=torch.ones(128, dtype=BF, device="cuda")), v)
    refused(cache.batch([0], [60], [8]), args(), v)                  # past the table's pages
    refused(cache.batch([1], [0], [8]), args(), v)                   # no such sequence
    with pytest.raises(ValueError):
        native.rope_args(q, k, qo, None, pos, t)                     # k_out may be left out of append_rope alone
    torch.cuda.synchronize()
    assert torch.equal(cache.pool, before) and cache.sync_status() == native.TSS_OK
    none = native.rope_args(q[:0], k[:0], qo[:0], None, pos[:0], t, to_pages=True)
    cache.append_rope(0, cache.batch([0], [0], [0]), none, v[:0])    # no rows: nothing to do
    assert torch.equal(cache.pool, before)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("way", ["no k_out", "k_out", "in place"])
def test_heads_that_turn_as_a_whole(dtype, norm, way):
    """128 dims, half layout, 16 bits, with runs that begin and end anywhere in a half page, values of all sizes, NaN and infinities."""
    first, n = (5, 63, 31, 40, 96, 0), (3, 2, 70, 33, 1, 32)
    lens, rows, hq, hk, d = [f + m for f, m in zip(first, n)], sum(n), 6, 3, 128
    one, two = (make(lens, hq, hk, d) for _ in range(2))
    q, k, v = (x.clone() for x in rows_of(rows, hq, hk, d, dtype, 12))
    k[7, 1] *= 1e-6
    k[9, 0] *= 500.0
    k[11, 2] = 0.0
    k[20, 1, 77], k[21, 2, 3] = float("nan"), float("inf")
    qg, kg = gains(d, dtype, 12) if norm else (None, None)
    t = table_of(128, 200)
    pos = torch.cat([torch.arange(f, f + m, device="cuda") for f, m in zip(first, n)]).to(torch.int32)
    qr, kr = torch.empty_like(q), torch.empty_like(k)
    native.qk_rope(native.rope_args(q, k, qr, kr, pos, t, q_gain=qg, k_gain=kg))
    batch = one.batch(range(6), first, n)
    two.append(0, batch, kr, v)
    qo = torch.empty_like(q)
    ko = {"no k_out": None, "k_out": torch.empty_like(k), "in place": k}[way]
    one.append_rope(0, batch, native.rope_args(q, k, qo, ko, pos, t, q_gain=qg, k_gain=kg, to_pages=True), v)
    assert one.sync_status() == native.TSS_OK and two.sync_status() == native.TSS_OK
    assert torch.equal(one.pool, two.pool) and torch.equal(qo, qr)
    if ko is not None:
        assert torch.equal(ko.view(torch.int16), kr.view(torch.int16))
    # without their pages the rows still reach q_out and k_out
    if way == "k_out":
        one.table[2, 0], one.table[3, 1] = -1, 10 ** 6
        before = one.pool.clone()
        ko.zero_()
        one.append_rope(0, batch, native.rope_args(q, k, qo, ko, pos, t, q_gain=qg, k_gain=kg, to_pages=True), v)
        assert one.sync_status() == native.TSS_ERR_DEVICE_CHECK
        assert torch.equal(one.pool, before) and torch.equal(ko.view(torch.int16), kr.view(torch.int16))
