"""What weights of one fp16 part cost outputs over many keys: bf16 outputs of blocks and groups of more than 8 rows of a KV head.

out = sum p v / sum p, v = s c + z.  A weight p s rounded to fp16 is off by d p s, |d| <= 2^-11 (half of fp16's step), of any sign
and apart from the other keys'.  With codes centred, v = s (c - 7.5) + (z + 7.5 s), that moves the output by sum d p s (c - 7.5), whose mean
square is at most W = (2^-11)^2 / 3 sum (p s (c - 7.5))^2, p normalised; the second term's sum is one of fp32.  With codes as they
are it would be sum d p s c, which over 64 dims' range of 15 s has six times the mean square and is not of the output's size
where many keys are averaged.
The sum over all outputs of (out - ref)^2 exceeds that of bf16's own roundings of ref by the weights' mean square alone, since the two
are apart: by at most 1.25 sum W (thousands of roundings come out otherwise: a twentieth of it or less), W's bound counting
every mantissa as 1 where the mean is half of that."""
import pytest
import torch

import paged_ref as R
from paper_2609_26100_gb300 import native, paged

pytestmark = pytest.mark.gpu


def tokens(c, seq, first, n, g):
    k, v = (torch.randn(n, c.n_kv_heads, c.head_dim, generator=g, device="cuda").bfloat16() for _ in range(2))
    c.append(0, c.batch([seq], [first], [n]), k, v)


def excess(c, seq, q, out, first, rows):
    """Sums over the outputs of rows of sequence seq: (out - ref)^2, bf16's own, W."""
    hk, d, gq, keys = c.n_kv_heads, c.head_dim, c.n_q_heads // c.n_kv_heads, first + rows
    k, v = (R.sequence_values(c.pool[0], c.table, seq, keys, hk, d, side) for side in (0, 1))
    blocks = c.pool[0].view(-1, hk, R.block_bytes(d))[c.table[seq, :-(-keys // 64)].long()]
    s, z = (R.params_of(blocks, d, 1)[..., i].double().permute(0, 2, 1, 3).reshape(-1, hk, d // 64)[:keys].repeat_interleave(64, -1) for i in (0, 1))
    centred = v - z - 7.5 * s
    total = [0.0, 0.0, 0.0]
    for h in range(c.n_q_heads):
        see = R.sees(first, rows, None, range(first, first + rows), 0, 0, "cuda")
        p = (q[:, h].double() @ k[:, h // gq].t() * d ** -0.5).masked_fill(~see, -torch.inf).softmax(-1)
        ref = p @ v[:, h // gq]
        w = p.square() @ centred[:, h // gq].square()
        for i, x in enumerate(((out[:, h].double() - ref).square(), (ref.bfloat16().double() - ref).square(), w * 2.0 ** -22 / 3)):
            total[i] += float(x.sum())
    return total


def holds(total):
    off, own, w = (sum(t[i] for t in total) for i in range(3))
    assert off - own <= 1.25 * w, (off, own, w, (off - own) / w)


@pytest.mark.parametrize("rows,hq,hk,d", [(16, 8, 8, 128), (9, 16, 8, 128), (16, 8, 8, 64), (12, 4, 1, 64)])
@pytest.mark.parametrize("first", [2000, 9000])
@pytest.mark.parametrize("spread", [0.0, 1.5])
def test_blocks(rows, hq, hk, d, first, spread):
    g = torch.Generator(device="cuda").manual_seed(first + rows)
    pages = paged.pages_for(first + rows)
    c = paged.Kv4Cache.allocate(n_layers=1, n_pages=pages, n_seqs=1, max_pages=pages, n_q_heads=hq, n_kv_heads=hk, head_dim=d)
    c.pages.reserve([0], [first + rows])
    tokens(c, 0, 0, first + rows, g)
    q = (torch.randn(rows, hq, d, generator=g, device="cuda") * spread).bfloat16()
    out = torch.empty_like(q)
    c.attention(0, c.batch([0], [first], [rows]), q, out)
    assert c.sync_status() == native.TSS_OK
    holds([excess(c, 0, q, out, first, rows)])


@pytest.mark.parametrize("beams,hq,hk,d", [(16, 8, 8, 128), (11, 16, 4, 128), (24, 16, 4, 128), (20, 8, 8, 64)])
@pytest.mark.parametrize("prompt", [2000, 9000])
@pytest.mark.parametrize("spread", [0.0, 1.5])
def test_shared_keys(beams, hq, hk, d, prompt, spread):
    g = torch.Generator(device="cuda").manual_seed(prompt + beams)
    pages = paged.pages_for(prompt + 1)
    c = paged.Kv4Cache.allocate(n_layers=1, n_pages=pages + 2 * beams, n_seqs=beams, max_pages=pages, n_q_heads=hq, n_kv_heads=hk, head_dim=d,
                                shared_rows=beams)
    c.pages.reserve([0], [prompt])
    tokens(c, 0, 0, prompt, g)
    c.pages.fork([0] * (beams - 1), list(range(1, beams)), [prompt] * (beams - 1))
    c.pages.reserve(list(range(beams)), [prompt + 1] * beams)
    for b in range(beams):
        tokens(c, b, prompt, 1, g)
    q = (torch.randn(beams, hq, d, generator=g, device="cuda") * spread).bfloat16()
    out = torch.empty_like(q)
    c.attention_shared(0, c.batch(list(range(beams)), [prompt] * beams, [1] * beams), c.groups([beams], [prompt]), q, out)
    assert c.sync_status() == native.TSS_OK and c.pages.sync_status() == native.TSS_OK
    holds([excess(c, b, q[b:b + 1], out[b:b + 1], prompt, 1) for b in range(beams)])
