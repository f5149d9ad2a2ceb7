"""Plain 64-bit references of the paged 4-bit cache's operators, written from the layout and formulas that
include/tss.h states."""
import math

import torch

PAGE, GROUP = 64, 64


def block_bytes(d):
    return PAGE * d + 512 * (d // GROUP)


def k_place(tok, dim, d):
    """Index of a K code (4-bit units) within its block."""
    g, t, x = dim // 64, dim % 64 // 16, dim % 16
    return tok * d + t * (16 * (d // 64)) + g * 16 + x


def v_place(tok, dim, d):
    half, r = tok // 32, tok % 32
    word = ((half * (d // 4) + dim // 4) * 4 + r % 8 // 2) * 4 + dim % 4
    return PAGE * d + word * 8 + r // 8 + 4 * (r % 2)


def codes_of(block, d, side):
    """[..., bytes] -> codes [..., 64, d] (int64)."""
    tok, dim = torch.meshgrid(torch.arange(PAGE, device=block.device), torch.arange(d, device=block.device), indexing="ij")
    at = (k_place if side == 0 else v_place)(tok, dim, d)
    return (block[..., at // 2].long() >> (4 * (at % 2))) & 15


def params_of(block, d, side):
    """[..., bytes] -> (s, z) [..., 64, groups, 2] (float16)."""
    g = d // GROUP
    p = block[..., PAGE * d:].contiguous().view(torch.float16)
    return p.reshape(*block.shape[:-1], 2, PAGE, g, 2)[..., side, :, :, :]


def block_values(block, d, side):
    p = params_of(block, d, side).double()
    s, z = (p[..., i].repeat_interleave(GROUP, -1) for i in (0, 1))
    return codes_of(block, d, side).double() * s + z


def sequence_values(pool, table, seq, n, heads, d, side):
    """Values [n][heads][d] in 64 bits of a sequence's first n tokens; pool [pages][bytes]."""
    pages = table[seq, :-(-n // PAGE)].long()
    blocks = pool.view(pool.shape[0], heads, -1)[pages]
    return block_values(blocks, d, side).permute(0, 2, 1, 3).reshape(-1, heads, d)[:n]


def quantised(x):
    """The definition on fp32 values [..., d]: (codes, s, z)."""
    x = x.float().unflatten(-1, (-1, GROUP))
    bad = ~torch.isfinite(x).all(-1)
    y = torch.where(torch.isfinite(x), x, 0.0)
    z = y.amin(-1).clamp(-65504, 65504).half()
    s = ((y.amax(-1) - z.float()) / 15).clamp(0, 65504).half()
    c = torch.where(s.float()[..., None] > 0, ((y - z.float()[..., None]) / s.float()[..., None]), 0.0).round().clamp(0, 15)
    s = torch.where(bad, torch.full_like(s, math.nan), s)
    return c, s, z


def stored(x):
    """What values [..., d] read back as, in 64 bits."""
    c, s, z = quantised(x)
    return (c.double() * s.double()[..., None] + z.double()[..., None]).flatten(-2)


def sees(first, n, mask, pos, window, sinks, device):
    """[n][first + n] visibility; mask: list of ancestor sets (ints) or None; pos: positions [n]."""
    j = torch.arange(first + n, device=device)
    if mask is None:
        block = torch.ones(n, n, dtype=torch.bool, device=device).tril()
    else:
        block = torch.tensor([[m >> i & 1 for i in range(n)] for m in mask], dtype=torch.bool, device=device).view(n, n)
    see = torch.cat([torch.ones(n, first, dtype=torch.bool, device=device), block], 1)
    if window:
        p = torch.tensor([max(int(x), first) for x in pos], device=device)
        where = torch.cat([j[:first], p])
        see &= (p[:, None] - where[None] < window) | (j[None] < sinks)
    return see


def attention(k, v, q, see, scale):
    """k, v [keys][kv heads][d], q [n][heads][d] in 64 bits; (out, lse); rows that see nothing: 0, -inf."""
    n, hq, d = q.shape
    g = hq // k.shape[1]
    out, lse = torch.zeros(n, hq, d, dtype=torch.float64, device=q.device), torch.full((n, hq), -math.inf, dtype=torch.float64, device=q.device)
    for i in range(n):
        keep = see[i].nonzero()[:, 0]
        if len(keep) == 0:
            continue
        for h in range(hq):
            s = k[keep, h // g] @ q[i, h] * scale
            lse[i, h] = torch.logsumexp(s, 0)
            out[i, h] = torch.softmax(s, 0) @ v[keep, h // g]
    return out, lse


def words(sets):
    """Ancestor sets (ints below 2^128) as int64 pairs."""
    signed = lambda x: x - (1 << 64) if x >> 63 else x  # noqa: E731
    return [[signed(x & (1 << 64) - 1), signed(x >> 64)] for x in sets]
