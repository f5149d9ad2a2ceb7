"""tss_qk_rope, tss_rope_table and tss_rope_frequencies against the formulas in 64 bits.

Tolerances.  An output is one rounding of an fp32 value: half the spacing of the type's numbers, at most
2^-8 (bf16: 8 significant bits, 2^-7 apart above 1), 2^-11 (fp16) or 2^-24 of its magnitude.  The fp32 part: the mean of squares of d values (relative error at most d 2^-24, halved
by the root), the root, quotient and products (each 2^-23), and the two products of the rotation, whose
result may cancel: so errors are held to the pair's magnitude |a| + |b|, (d / 2 + 8) 2^-23 of it."""
import math

import pytest
import torch

from paper_2609_26100_gb300 import native

pytestmark = pytest.mark.gpu
HALF_ULP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}


def reference(x, gain, eps, cs, rot, inter):
    """x [n][h][d] double, cs [n][rot / 2][2]: (result, magnitude of the pair each value comes from)."""
    if gain is not None:
        x = x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * gain
    i = torch.arange(rot // 2, device=x.device)
    a, b = (2 * i, 2 * i + 1) if inter else (i, i + rot // 2)
    c, s = cs[:, None, :, 0], cs[:, None, :, 1]
    y, mag = x.clone(), x.abs()
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    m = x[..., a].abs() + x[..., b].abs()
    mag[..., a], mag[..., b] = m, m
    return y, mag


@pytest.mark.parametrize("d,rot,inter", [(128, 128, False), (128, 64, True), (64, 64, True), (64, 32, False), (16, 16, False),
                                         (80, 48, True), (96, 96, False), (256, 256, False), (256, 16, True), (128, 0, False),
                                         (32, 32, True)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("rows,hq,hk,norm", [(1, 1, 1, True), (5, 7, 3, True), (67, 8, 2, False), (130, 40, 8, True)])
def test_norm_and_rotation(d, rot, inter, dtype, rows, hq, hk, norm):
    g = torch.Generator(device="cuda").manual_seed(d * 7 + rot + rows)
    fused = torch.randn(rows, hq + 2 * hk, d, generator=g, device="cuda").to(dtype)
    q, k = fused[:, :hq], fused[:, hq:hq + hk]  # slices: the row stride is that of the fused rows
    keep = fused.clone()
    gains = [(1 + 0.3 * torch.randn(d, generator=g, device="cuda")).to(dtype) if norm else None for _ in range(2)]
    table = torch.randn(300, rot // 2, 2, generator=g, device="cuda") if rot else None
    pos = torch.randint(0, 300, (rows,), generator=g, device="cuda", dtype=torch.int32)
    qo, ko = torch.empty(rows, hq, d, dtype=dtype, device="cuda"), torch.empty(rows, hk, d, dtype=dtype, device="cuda")
    native.qk_rope(native.rope_args(q, k, qo, ko, pos, table, q_gain=gains[0], k_gain=gains[1], eps=1e-5, interleaved=inter))
    assert torch.equal(fused, keep)
    cs = table.double()[pos.long()] if rot else torch.zeros(rows, 0, 2, dtype=torch.float64, device="cuda")
    for x, y, gain in ((q, qo, gains[0]), (k, ko, gains[1])):
        ref, mag = reference(x.double(), None if gain is None else gain.double(), 1e-5, cs, rot, inter)
        scale = cs.abs().sum(-1).amax(-1)[:, None, None].clamp(min=1) if rot else 1.0
        # (fp16 below its normal range: half of 2^-24)
        bound = ref.abs() * HALF_ULP[dtype] * 1.01 + mag * scale * (d / 2 + 8) * 2.0 ** -23 + (2.0 ** -25 if dtype == torch.float16 else 0)
        assert ((y.double() - ref).abs() <= bound).all()
    # in place over the slices, the same bits
    native.qk_rope(native.rope_args(q, k, q, k, pos, table, q_gain=gains[0], k_gain=gains[1], eps=1e-5, interleaved=inter))
    assert torch.equal(q, qo) and torch.equal(k, ko) and torch.equal(fused[:, hq + hk:], keep[:, hq + hk:])


def test_one_side_and_no_rows():
    x = torch.randn(3, 4, 64, device="cuda")
    table, pos = torch.randn(9, 32, 2, device="cuda"), torch.tensor([0, 8, 3], dtype=torch.int32, device="cuda")
    both = [torch.empty_like(x) for _ in range(2)]
    native.qk_rope(native.rope_args(x, x, *both, pos, table))
    one = torch.empty_like(x)
    native.qk_rope(native.rope_args(None, x, None, one, pos, table))
    assert torch.equal(one, both[0]) and torch.equal(one, both[1])
    native.qk_rope(native.rope_args(x, None, one, None, pos, table))
    assert torch.equal(one, both[0])
    native.qk_rope(native.rope_args(x[:0], None, one[:0], None, pos[:0], table))


def test_a_norm_on_one_side_alone():
    x = torch.randn(9, 4, 128, device="cuda")
    gain = torch.rand(128, device="cuda")
    qo, ko = torch.empty_like(x), torch.empty_like(x)
    native.qk_rope(native.rope_args(x, x, qo, ko, None, None, k_gain=gain, eps=0.0))
    assert torch.equal(qo, x)
    ref = x.double() / x.double().square().mean(-1, keepdim=True).sqrt() * gain.double()
    assert ((ko.double() - ref).abs() <= ref.abs() * 72 * 2.0 ** -23).all()


def test_a_position_outside_the_table_is_recorded():
    x = torch.randn(3, 2, 64, device="cuda")
    table = torch.randn(5, 32, 2, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got, want = torch.empty_like(x), torch.empty_like(x)
    native.qk_rope(native.rope_args(x, None, got, None, torch.tensor([-1, 2, 5], dtype=torch.int32, device="cuda"), table, status=status))
    assert int(status) == native.TSS_ERR_DEVICE_CHECK
    native.qk_rope(native.rope_args(x, None, want, None, torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda"), table))
    assert torch.equal(got, want)


def test_another_stream():
    x = torch.randn(64, 8, 128, device="cuda", dtype=torch.bfloat16)
    table, pos = torch.randn(64, 64, 2, device="cuda"), torch.arange(64, dtype=torch.int32, device="cuda")
    want, got = torch.empty_like(x), torch.empty_like(x)
    args = native.rope_args(x, None, want, None, pos, table)
    native.qk_rope(args)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        native.qk_rope(native.rope_args(x, None, got, None, pos, table))
    s.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(want, got)


@pytest.mark.parametrize("kind", sorted(native.ROPE_KINDS))
def test_table(kind):
    f, a = native.rope_frequencies(64, 10000.0, kind, 8.0, 4096.0)
    table = torch.empty(40001, 32, 2, device="cuda")
    native.rope_table(f, table, a)
    angle = torch.arange(40001, dtype=torch.float64)[:, None] * torch.tensor(f, dtype=torch.float64)
    ref = torch.stack([angle.cos(), angle.sin()], -1) * a
    # one rounding to fp32 (values up to `a`, below 2), and the doubles' own angle error, 4e4 2^-53
    assert (table.cpu().double() - ref).abs().max() <= 2.0 ** -24 * max(1.0, a) * 1.01 + 1e-11


def bad_args(**change):
    x = torch.randn(2, 2, 64, device="cuda", dtype=torch.bfloat16)
    a = native.rope_args(x, x, torch.empty_like(x), torch.empty_like(x), torch.zeros(2, dtype=torch.int32, device="cuda"),
                         torch.zeros(4, 32, 2, device="cuda"), q_gain=torch.ones(64, device="cuda", dtype=torch.bfloat16))
    for name, value in change.items():
        setattr(a, name, value(getattr(a, name)) if callable(value) else value)
    return a


@pytest.mark.parametrize("change", [
    {"n_rows": -1}, {"head_dim": 72}, {"head_dim": 272}, {"rot_dim": 24}, {"rot_dim": 80}, {"dtype": 3}, {"dtype": -1},
    {"q": None}, {"k_out": None}, {"q": lambda p: p + 2}, {"q_out": lambda p: p + 8}, {"q_gain": lambda p: p + 2},
    {"q_stride": 64}, {"k_stride": 129}, {"k_out_stride": 0}, {"table": None}, {"positions": None}, {"max_positions": 0},
    {"eps": -1.0}, {"eps": math.nan}, {"n_q_heads": -1}, {"table": lambda p: p + 4}])
def test_refusals(change):
    with pytest.raises(native.TssError) as e:
        native.qk_rope(bad_args(**change))
    assert e.value.status == native.TSS_ERR_INVALID_ARG
    native.qk_rope(bad_args())  # and the next call works
    torch.cuda.synchronize()
