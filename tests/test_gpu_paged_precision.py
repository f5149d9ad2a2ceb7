"""How many bits the paged attention's weights keep, for every variant of its kernels.

out = sum p (s c + z) / sum p over the keys that a row sees, p their softmax weights.  M = sum p (s c + |z|) / sum p is what
is summed, so errors of the sums are measured by it, each dim by its own group's s and z:
  * weights p s as two fp16 parts: 2^-22 of themselves, and 2^-21 each at least (the second part's last place, four bits up
    for odd codes) in units where a row's largest of the group, W, is 2^6 or more: 15 2^-27 W a key for codes up to 15;
  * 2^x: 2^-22, twice (it is in both sums);
  * the tensor cores' fp32 sums, which cut off what passes their end: 2^-22 an MMA, fewer than 2^5 of them in a run here;
  * scores: 2^-21 of A = log2(e) scale max_key sum_dims |q| (s c + |z|), the magnitude that they are summed of, times
    2 ln 2 for what it does to p in both sums;
together under (2^-16 + 2^-20 A) M + 15 2^-27 keys W; and the output's own half ulp: 2^-11 of it for fp16 (2^-25 at least),
2^-8 for bf16.  One part of 11 bits instead of two is off by 2^-13 of each weight on average, which few keys of equal
weight and mixed signs show where they cancel: bf16 outputs of blocks of more than 8 rows are held to that (2^-11 M)."""
import math

import pytest
import torch

import paged_ref as R
from paper_2609_26100_gb300 import native, paged

pytestmark = pytest.mark.gpu


def make(keys, hq, hk, d, group_scale, seed):
    """A cache of one sequence of random keys; V's second 64 dims times group_scale, or (None) each token's groups by powers
    of ten of their own, some of them zero.  (cache, k, v, (s c, z, s) of both, generator)"""
    pages = -(-keys // 64)
    c = paged.Kv4Cache.allocate(n_layers=1, n_pages=pages + 1, n_seqs=1, max_pages=pages + 1, n_q_heads=hq, n_kv_heads=hk, head_dim=d)
    c.pages.reserve([0], [keys])
    g = torch.Generator(device="cuda").manual_seed(seed)
    k, v = (torch.randn(keys, hk, d, generator=g, device="cuda") for _ in range(2))
    if group_scale is None:
        up = 10.0 ** (torch.rand(keys, hk, d // 64, generator=g, device="cuda") * 9 - 6)
        up[torch.rand(up.shape, generator=g, device="cuda") < 0.05] = 0.0
        v *= up.repeat_interleave(64, -1)
    else:
        v[..., 64:] *= group_scale
    c.append(0, c.batch([0], [0], [keys]), k, v)
    k, v = (R.sequence_values(c.pool[0], c.table, 0, keys, hk, d, side) for side in (0, 1))
    blocks = c.pool[0].view(-1, hk, R.block_bytes(d))[c.table[0, :pages].long()]
    part = []
    for side in (0, 1):
        s, z = (R.params_of(blocks, d, side)[..., i].double().permute(0, 2, 1, 3).reshape(-1, hk, d // 64)[:keys] for i in (0, 1))
        z = z.repeat_interleave(64, -1)
        part.append(((k, v)[side] - z, z, s))
    return c, k, v, part, g


def sums(part, k, q, see, scale):
    """In 64 bits, [rows][heads][d]: sum p s c and sum p z (p normalised), M, W; [rows][heads]: A; and sum p s c with each
    weight p s rounded to fp16 once, its row's largest (of the group) between 2^6 and 2^7."""
    gq = q.shape[1] // k.shape[1]
    kh = k.repeat_interleave(gq, 1)
    p = torch.einsum("nhd,shd->nhs", q, kh).mul_(scale).masked_fill_(~see[:, None], -math.inf).softmax(-1)
    (kc, kz, _), (vc, vz, vs) = [[x.repeat_interleave(gq, 1) for x in side] for side in part]
    code, zero, mag = (torch.einsum("nhs,shd->nhd", p, x) for x in (vc, vz, vc.abs() + vz.abs()))
    a = torch.einsum("nhd,shd->nhs", q.abs(), kc.abs() + kz.abs()).masked_fill_(~see[:, None], 0).amax(-1) * scale * math.log2(math.e)
    once, most = torch.empty_like(code), torch.empty_like(code)
    for i in range(vs.shape[2]):
        s, dims = vs[..., i], slice(64 * i, 64 * i + 64)
        w = p * s.t()[None]
        top = w.amax(-1, keepdim=True)
        up = 2.0 ** (7 - torch.ceil(torch.log2(top)))
        unit = torch.where(s[..., None] > 0, vc[..., dims] / s[..., None], 0.0)
        once[..., dims] = torch.einsum("nhs,shd->nhd", (w * up).half().double() / up, unit)
        most[..., dims] = top
    return code, zero, mag, most, a, once


CASES = [(1, 2, 2, 64), (1, 2, 2, 128), (5, 4, 4, 128), (2, 8, 2, 64), (12, 2, 2, 64), (12, 4, 4, 128), (40, 2, 1, 64), (20, 4, 2, 128),
         (60, 2, 2, 128), (30, 8, 2, 128), (100, 4, 2, 64), (128, 4, 4, 128)]


def check(dtype, rows, hq, hk, d, keys, qscale, group_scale, window=0, sinks=0):
    first = keys
    c, k, v, part, g = make(first + rows, hq, hk, d, group_scale, rows + keys)
    q = (torch.randn(rows, hq, d, generator=g, device="cuda") * qscale).to(dtype)
    out, lse = torch.empty_like(q), torch.empty(rows, hq, device="cuda")
    scale = d ** -0.5
    c.attention(0, c.batch([0], [first], [rows]), q, out, lse=lse, scale=scale, window=window, sinks=sinks)
    assert c.sync_status() == native.TSS_OK
    see = R.sees(first, rows, None, range(first, first + rows), window, sinks, "cuda")
    code, zero, mag, most, a, once = sums(part, k, q.double(), see, scale)
    ref = code + zero
    two = dtype == torch.float16 or rows * hq // hk <= 8
    half_ulp = ref.abs() * 2.0 ** -11 + 2.0 ** -25 if dtype == torch.float16 else ref.abs() * 2.0 ** -8
    bound = half_ulp + mag * ((2.0 ** -16 if two else 2.0 ** -11) + 2.0 ** -20 * a[..., None]) + 15 * 2.0 ** -27 * (first + rows) * most
    off = (out.double() - ref).abs() / bound
    worst = [float(off[..., i:i + 64].amax()) for i in range(0, d, 64)]
    assert max(worst) <= 1, worst
    return once, code, bound


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,hq,hk,d", CASES)
@pytest.mark.parametrize("keys,qscale", [(40, 0.01), (300, 0.01), (700, 3.0)])
@pytest.mark.parametrize("ratio", [1.0, 1e-4, 1e-6, 1e4])
def test_bits_of_the_weights(dtype, rows, hq, hk, d, keys, qscale, ratio):
    if d == 64 and ratio != 1.0:
        pytest.skip("one group")
    once, code, bound = check(dtype, rows, hq, hk, d, keys, qscale, ratio)
    # the bound sees one part where two are promised (where there are outputs enough, and their own rounding is fine enough)
    if dtype == torch.float16 and keys == 40 and ratio == 1.0 and rows * hq >= 40:
        assert ((once - code).abs() > bound).any()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,hq,hk,d", CASES)
@pytest.mark.parametrize("keys,qscale", [(100, 0.01), (900, 0.3), (800, 3.0)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (150, 3)])
def test_scales_that_differ_by_token_and_group(dtype, rows, hq, hk, d, keys, qscale, window, sinks):
    """References of the groups rise apart and together from page to page, and under a window at different pages for each row."""
    check(dtype, rows, hq, hk, d, keys, qscale, None, window, sinks)


@pytest.mark.parametrize("rows,hq,hk,d", [(1, 4, 4, 128), (6, 4, 2, 128), (20, 4, 2, 64), (61, 8, 2, 128)])
def test_two_runs_give_the_same_bits(rows, hq, hk, d):
    """Many CTAs share the items; whichever arrives last joins in the same order."""
    first = 6000
    c, *_, g = make(first + rows, hq, hk, d, 1.0, 5)
    q = torch.randn(rows, hq, d, generator=g, device="cuda").bfloat16()
    batch = c.batch([0], [first], [rows])
    want, want_lse = torch.empty_like(q), torch.empty(rows, hq, device="cuda")
    c.attention(0, batch, q, want, lse=want_lse)
    for _ in range(20):
        got, lse = torch.full_like(q, 9.0), torch.zeros(rows, hq, device="cuda")
        c.attention(0, batch, q, got, lse=lse)
        assert torch.equal(got, want) and torch.equal(lse, want_lse)
    assert c.sync_status() == native.TSS_OK
