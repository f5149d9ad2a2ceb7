"""Operators around a paged 4-bit KV cache: head norms with rotary positions, appending to the cache,
attention over it, and the bookkeeping of its pages.

Each is computed twice: in its plain form, elementary torch operations in 32 bits, and (own) by the
framework's kernels through the calls that a program makes.  exact() is the definition in 64 bits.

The cache.  A sequence's tokens lie in pages of 64, whose ids its row of the page table lists.  A page
holds a block for each KV head: K codes, V codes, K parameters, V parameters.  64 neighbouring dims of a
token's head share a scale s and a minimum z (16-bit floats); a code c of 4 bits stands for s c + z.
  K codes: by token; within a token 16-dim units, for each quarter t of a group, of every group in turn.
  V codes: 32-bit words of 8 tokens of one dim: by 32-token half, 4 dims, t, dim within the 4; nibble
           b + 4 i of word t is token 8 b + 2 t + i of the half.
  parameters: by token and group, (s, z).
"""
import math
import random

import torch

own = False
PAGE = 64
GROUP = 64
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def listed():
    return [
        # one user's chain of drafts at the 7B shape, norms on: launches and latency are all there is
        {"name": "rope_chain", "kind": "rope", "rows": 6, "hq": 32, "hk": 32, "d": 128, "rot": 128, "inter": False,
         "norm": True, "dtype": "bf16", "ctx": 1024, "factor": 1.0},
        # eight draft trees with grouped heads, half of each head rotated in neighbouring pairs, positions stretched
        {"name": "rope_trees", "kind": "rope", "rows": 488, "hq": 40, "hk": 8, "d": 128, "rot": 64, "inter": True,
         "norm": False, "dtype": "f16", "ctx": 60000, "factor": 8.0},
        # a pass over a long prompt
        {"name": "rope_prompt", "kind": "rope", "rows": 4096, "hq": 32, "hk": 32, "d": 128, "rot": 128, "inter": False,
         "norm": True, "dtype": "bf16", "ctx": 0, "factor": 1.0},
        # the new rows of a step of 16 long requests (7B), and a look back at what they stand beside
        {"name": "append_step", "kind": "append", "ctx": ",".join(str(1000 + 997 * i) for i in range(16)),
         "n": ",".join(["9"] * 16), "hk": 32, "d": 128, "dtype": "bf16", "back": 33},
        # prompts of ragged lengths at the 13B shape, some on top of a context
        {"name": "append_prompt", "kind": "append", "ctx": "0,77,512,4095", "n": "4096,2051,1,1023", "hk": 40, "d": 128,
         "dtype": "bf16", "back": 0},
        # one user, one token: latency
        {"name": "attn_single", "kind": "attn", "ctx": "1024", "n": "1", "hq": 32, "hk": 32, "d": 128, "dtype": "bf16",
         "window": 0, "sinks": 0, "tree": False},
        # eight requests of mixed lengths with chains of five drafts (13B)
        {"name": "attn_chains", "kind": "attn", "ctx": "512,871,1304,1777,2290,2906,3511,4096", "n": "6,6,6,6,6,6,6,6",
         "hq": 40, "hk": 40, "d": 128, "dtype": "bf16", "window": 0, "sinks": 0, "tree": False},
        # 16 requests of 16384 tokens, chains of eight drafts (7B): the cache's bytes are the cost
        {"name": "attn_long", "kind": "attn", "ctx": ",".join(["16384"] * 16), "n": ",".join(["9"] * 16), "hq": 32, "hk": 32,
         "d": 128, "dtype": "bf16", "window": 0, "sinks": 0, "tree": False},
        # single tokens far into long texts: a window of 4096 and the first tokens, grouped heads
        {"name": "attn_window", "kind": "attn", "ctx": ",".join(str(20000 + 1531 * i) for i in range(32)),
         "n": ",".join(["1"] * 32), "hq": 32, "hk": 8, "d": 128, "dtype": "f16", "window": 4096, "sinks": 4, "tree": False},
        # draft trees of 60 nodes and their root, grouped heads: many rows share the cache's bytes
        {"name": "attn_trees", "kind": "attn", "ctx": "2048,3333,8000,5000", "n": "61,61,61,61", "hq": 32, "hk": 8, "d": 128,
         "dtype": "bf16", "window": 0, "sinks": 0, "tree": True},
        # hypotheses dropped and forked from better ones: shared pages, a copied tail in every layer
        {"name": "pages_fork", "kind": "fork", "layers": 8, "pages": 512, "elems": 32768, "seqs": 24, "forks": 12,
         "tokens": "1000,333,64,2050", "maxp": 64},
        # a pool thinned out by requests that ended, made dense again
        {"name": "pages_compact", "kind": "compact", "layers": 2, "pages": 4096, "elems": 65536, "seqs": 64, "live": 1800,
         "moves": 900, "maxp": 128},
    ]


def draw(rng):
    def log_int(lo, hi):
        return min(hi, int(round(lo * (hi / lo) ** rng.random())))

    kind = rng.choice(("rope", "rope", "append", "append", "attn", "attn", "attn", "attn", "fork", "compact"))
    d = rng.choice((64, 128, 128))
    hk = rng.choice((4, 8, 32, 40))
    group = rng.choice((1, 1, 2, 4)) if hk <= 8 else 1
    dtype = rng.choice(("bf16", "bf16", "f16"))
    if kind == "rope":
        return {"kind": kind, "rows": log_int(1, 4000), "hq": hk * group, "hk": hk, "d": d, "rot": rng.choice((d, d, d // 2)),
                "inter": rng.random() < 0.4, "norm": rng.random() < 0.6, "dtype": dtype, "ctx": log_int(1, 60000),
                "factor": rng.choice((1.0, 4.0, 8.0))}
    if kind == "append":
        b = log_int(1, 16)
        top = max(2, 7000 // b)
        return {"kind": kind, "ctx": ",".join(str(rng.randrange(8000)) for _ in range(b)),
                "n": ",".join(str(log_int(1, top)) for _ in range(b)), "hk": hk, "d": d, "dtype": dtype,
                "back": rng.choice((0, 33, 65))}
    if kind == "attn":
        b = log_int(1, 32)
        top = max(64, 160000 // b // max(1, hk // 8))
        n = rng.choice((1, 1, 2, 6, 9, 16, 33, 61, 128))
        n = min(n, max(1, 512 // b))
        tree = n > 4 and rng.random() < 0.5
        window = rng.choice((0, 0, 0, log_int(64, 8192)))
        return {"kind": kind, "ctx": ",".join(str(log_int(1, min(top, 40000))) for _ in range(b)),
                "n": ",".join(str(n if rng.random() < 0.7 else rng.randrange(1, n + 1)) for _ in range(b)), "hq": hk * group,
                "hk": hk, "d": d, "dtype": dtype, "window": window, "sinks": rng.choice((0, 4, 70)) if window else 0,
                "tree": tree}
    if kind == "fork":
        f = log_int(1, 12)
        return {"kind": kind, "layers": rng.randrange(1, 9), "pages": rng.randrange(300, 513), "elems": 4096 * rng.randrange(1, 9),
                "seqs": 24, "forks": f, "tokens": ",".join(str(log_int(1, 3000)) for _ in range(4)), "maxp": 64}
    pages = log_int(64, 4096)
    live = max(4, int(pages * rng.uniform(0.2, 0.7)))
    return {"kind": kind, "layers": rng.randrange(1, 3), "pages": pages, "elems": 8192 * rng.randrange(1, 9), "seqs": 64,
            "live": live, "moves": max(1, int(min(live, pages - live) * rng.uniform(0.1, 0.9))), "maxp": 4096}


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------
def ints(text):
    return [int(x) for x in text.split(",")]


def generator(seed, tag):
    return torch.Generator(device="cuda").manual_seed((seed * 1000003 + sum(ord(c) * 131 ** i for i, c in enumerate(tag))) % (1 << 62))


def normal(seed, tag, shape, dtype=torch.float32, std=1.0):
    return (torch.randn(shape, generator=generator(seed, tag), device="cuda") * std).to(dtype)


def permutation(seed, tag, n):
    return torch.randperm(n, generator=generator(seed, tag), device="cuda")


def block_bytes(d):
    return PAGE * d + PAGE * (d // GROUP) * 8


def pack(kc, vc, kp, vp):
    """Codes [..., 64, d] (uint8) and parameters [..., 64, groups, 2] (float16) to blocks [..., bytes]."""
    *lead, _, d = kc.shape
    g = d // GROUP
    k = kc.reshape(*lead, PAGE, g, 4, 16).transpose(-3, -2).reshape(*lead, PAGE * d // 2, 2)
    v = vc.reshape(*lead, 2, 4, 4, 2, d // 4, 4)  # half, b, t, i, dims / 4, dim
    n = len(lead)
    v = v.permute(*range(n), n, n + 4, n + 2, n + 5, n + 3, n + 1).reshape(*lead, PAGE * d // 2, 2)
    params = [p.contiguous().view(torch.uint8).reshape(*lead, PAGE * g * 4) for p in (kp, vp)]
    return torch.cat([k[..., 0] + 16 * k[..., 1], v[..., 0] + 16 * v[..., 1], *params], -1)


def unpack(blocks, d):
    """pack() backwards."""
    *lead, _ = blocks.shape
    g, half = d // GROUP, PAGE * d // 2
    n = len(lead)

    def nibbles(x):
        return torch.stack([x & 15, x >> 4], -1)

    kc = nibbles(blocks[..., :half]).reshape(*lead, PAGE, 4, g, 16).transpose(-3, -2).reshape(*lead, PAGE, d)
    v = nibbles(blocks[..., half:2 * half]).reshape(*lead, 2, d // 4, 4, 4, 2, 4)  # half, dims / 4, t, dim, i, b
    vc = v.permute(*range(n), n, n + 5, n + 2, n + 4, n + 1, n + 3).reshape(*lead, PAGE, d)
    params = blocks[..., 2 * half:].contiguous().view(torch.float16).reshape(*lead, 2, PAGE, g, 2)
    return kc, vc, params[..., 0, :, :, :], params[..., 1, :, :, :]


def values(codes, params, dtype=torch.float32):
    s, z = (params[..., i].to(dtype).repeat_interleave(GROUP, -1) for i in (0, 1))
    return codes.to(dtype) * s + z


def filled(seed, n_pages, heads, d):
    """A pool [pages][bytes] of what quantised keys and values look like: codes around the middle, a scale
    and a minimum for every token and group."""
    pool = torch.empty(n_pages, heads * block_bytes(d), dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 26) // (heads * PAGE * d))
    for a in range(0, n_pages, step):
        m = min(step, n_pages - a)
        codes = [(normal(seed, "codes%d.%d" % (i, a), (m, heads, PAGE, d)) * 3.2 + 7.5).round_().clamp_(0, 15).to(torch.uint8)
                 for i in (0, 1)]
        params = []
        for i in (0, 1):
            s = (normal(seed, "s%d.%d" % (i, a), (m, heads, PAGE, d // GROUP)) * 0.15).exp() * (0.31, 0.2)[i]
            z = -7.5 * s + normal(seed, "z%d.%d" % (i, a), s.shape) * 0.1
            params.append(torch.stack([s, z], -1).to(torch.float16))
        pool[a:a + m] = pack(*codes, *params).reshape(m, -1)
    return pool


def tables(seed, lens):
    """Page table of sequences of the given lengths, their pages strewn over the pool: (table, pages of the pool)."""
    need = [-(-n // PAGE) for n in lens]
    ids = permutation(seed, "pages", sum(need) + 3).to(torch.int32)
    table = torch.full((len(lens), max(need)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = ids[at:at + n]
        at += n
    return table, sum(need) + 3


def parents(case, b, n):
    """A draft tree: every node hangs from one of the four before it that came last."""
    rng = random.Random("%s.%d" % (case["ctx"], b))
    return [-1] + [max(0, i - 1 - rng.randrange(4)) for i in range(1, n)]


def tree(case, b, n):
    """(ancestor-or-self sets as whole numbers, depths) of request b's block."""
    sets, depth = [], []
    for i, p in enumerate(parents(case, b, n) if case["tree"] else range(-1, n - 1)):
        sets.append((sets[p] if p >= 0 else 0) | 1 << i)
        depth.append(depth[p] + 1 if p >= 0 else 0)
    return sets, depth


def prepare(case, seed):
    """What a program has in hand before the call."""
    return {"rope": prepare_rope, "append": prepare_append, "attn": prepare_attn, "fork": prepare_fork,
            "compact": prepare_compact}[case["kind"]](case, seed)


def prepare_rope(case, seed):
    n, d, rot, dtype = case["rows"], case["d"], case["rot"], DTYPES[case["dtype"]]
    # the table a model keeps: base 10000, frequencies divided by the factor beyond the first quarter (long waves)
    inv = 10000.0 ** (-torch.arange(rot // 2, dtype=torch.float64, device="cuda") * 2 / rot)
    inv[rot // 8:] /= case["factor"]
    angle = torch.arange(case["ctx"] + n, dtype=torch.float64, device="cuda")[:, None] * inv
    scale = 0.1 * math.log(case["factor"]) + 1.0
    fused = normal(seed, "qkv", (n, case["hq"] + 2 * case["hk"], d), dtype)  # q, k and v rows of one projection
    s = {"case": case, "q": fused[:, :case["hq"]], "k": fused[:, case["hq"]:case["hq"] + case["hk"]],
         "table": (torch.stack([angle.cos(), angle.sin()], -1) * scale).float(),
         "positions": (case["ctx"] + torch.arange(n, device="cuda")).to(torch.int32)}
    for x in ("q", "k"):
        s[x + "_gain"] = (1 + normal(seed, x + "gain", (d,), std=0.1)).to(dtype) if case["norm"] else None
    if own:
        from paper_2609_26100_gb300 import native

        s["q_out"], s["k_out"] = (torch.empty(s[x].shape, dtype=dtype, device="cuda") for x in ("q", "k"))
        s["args"] = native.rope_args(s["q"], s["k"], s["q_out"], s["k_out"], s["positions"], s["table"], q_gain=s["q_gain"],
                                     k_gain=s["k_gain"], eps=1e-6, interleaved=case["inter"])
    return s


def prepare_append(case, seed):
    ctx, n, hk, d, dtype = ints(case["ctx"]), ints(case["n"]), case["hk"], case["d"], DTYPES[case["dtype"]]
    table, n_pages = tables(seed, [c + m for c, m in zip(ctx, n)])
    s = {"case": case, "pool": filled(seed, n_pages, hk, d), "table": table, "seqs": list(range(len(ctx))), "ctx": ctx, "n": n,
         "first": [max(0, c - case["back"]) for c in ctx]}
    fused = normal(seed, "kv", (sum(n), 2 * hk, d), dtype)
    fused[:, :hk, ::17] *= 4.0  # channels that stand out, as keys have them
    s["k"], s["v"] = fused[:, :hk], fused[:, hk:]
    s["look"] = [c + m - f for c, m, f in zip(ctx, n, s["first"])]
    if own:
        from paper_2609_26100_gb300 import paged

        s["cache"] = paged.Kv4Cache(s["pool"][None], table, n_q_heads=hk, n_kv_heads=hk, head_dim=d)
        s["batch"] = s["cache"].batch(s["seqs"], ctx, n)
        s["reads"] = s["cache"].batch(s["seqs"], s["first"], s["look"])
        s["k_back"], s["v_back"] = (torch.empty(sum(s["look"]), hk, d, dtype=dtype, device="cuda") for _ in range(2))
    return s


def prepare_attn(case, seed):
    ctx, n, hq, d, dtype = ints(case["ctx"]), ints(case["n"]), case["hq"], case["d"], DTYPES[case["dtype"]]
    table, n_pages = tables(seed, [c + m for c, m in zip(ctx, n)])
    q = normal(seed, "q", (sum(n), hq, d), dtype, 2.0)
    sets = [tree(case, b, m) for b, m in enumerate(n)]
    words = [[(x >> 64 * i & (1 << 64) - 1) - (x >> 64 * i + 63 & 1) * (1 << 64) for i in (0, 1)] for a, _ in sets for x in a]
    s = {"case": case, "pool": filled(seed, n_pages, case["hk"], d), "table": table, "seqs": list(range(len(ctx))), "ctx": ctx,
         "n": n, "q": q, "mask": torch.tensor(words, dtype=torch.int64, device="cuda") if case["tree"] else None,
         "positions": torch.tensor([c + x for c, (_, dep) in zip(ctx, sets) for x in dep], dtype=torch.int32, device="cuda")}
    if own:
        from paper_2609_26100_gb300 import paged

        s["cache"] = paged.Kv4Cache(s["pool"][None], table, n_q_heads=hq, n_kv_heads=case["hk"], head_dim=d)
        s["batch"] = s["cache"].batch(s["seqs"], ctx, n)
        s["out"] = torch.empty_like(q)
        s["lse"] = torch.empty(q.shape[:2], dtype=torch.float32, device="cuda")
    return s


def prepare_fork(case, seed):
    lens = ints(case["tokens"])
    need = [-(-x // PAGE) for x in lens]
    table = torch.full((case["seqs"], case["maxp"]), -1, dtype=torch.int32, device="cuda")
    held = torch.zeros(case["seqs"], dtype=torch.int32, device="cuda")
    refs = torch.zeros(case["pages"], dtype=torch.int32, device="cuda")
    ids, at = permutation(seed, "pages", case["pages"]).to(torch.int32), 0
    for b, m in enumerate(need):
        table[b, :m], held[b] = ids[at:at + m], m
        at += m
    refs[ids[:at].long()] = 1
    dst = list(range(case["seqs"] - case["forks"], case["seqs"]))
    src = [i % len(lens) for i in range(case["forks"])]
    s = {"case": case, "pool": normal(seed, "pool", (case["layers"], case["pages"], case["elems"]), torch.bfloat16), "table": table,
         "held": held, "refs": refs, "src": src, "dst": dst, "tokens": [lens[i] for i in src]}
    if own:
        from paper_2609_26100_gb300 import paged

        s["pages"] = paged.PagePool(s["pool"], table, held, refs)
    return s


def prepare_compact(case, seed):
    pages, live, moves = case["pages"], case["live"], case["moves"]
    low = permutation(seed, "low", live)[:live - moves]
    high = live + permutation(seed, "high", pages - live)[:moves]
    ids = torch.cat([low, high])[permutation(seed, "mix", live)].to(torch.int32)
    table = torch.full((case["seqs"], case["maxp"]), -1, dtype=torch.int32, device="cuda")
    rng = random.Random(seed)
    cuts = sorted(rng.randrange(live + 1) for _ in range(case["seqs"] - 1))
    sizes = [min(b - a, case["maxp"] - 2) for a, b in zip([0] + cuts, cuts + [live])]
    spare = live - sum(sizes)
    for i in range(len(sizes)):  # what a cut would have put over a row's end
        more = min(spare, case["maxp"] - 2 - sizes[i])
        sizes[i], spare = sizes[i] + more, spare - more
    at = 0
    for b, m in enumerate(sizes):
        table[b, :m] = ids[at:at + m]
        at += m
    refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
    refs[ids.long()] = 1
    first = max(range(len(sizes)), key=lambda i: sizes[i])  # two of its pages are shared with every third sequence
    for b in range(0, len(sizes), 3):
        if b != first and sizes[first] >= 2:
            table[b, sizes[b]:sizes[b] + 2] = table[first, :2]
            refs[table[first, :2].long()] += 1
            sizes[b] += 2
    s = {"case": case, "pool": normal(seed, "pool", (case["layers"], pages, case["elems"]), torch.bfloat16), "table": table,
         "held": torch.tensor(sizes, dtype=torch.int32, device="cuda"), "refs": refs}
    if own:
        from paper_2609_26100_gb300 import paged

        s["pages"] = paged.PagePool(s["pool"], table, s["held"], refs)
        s["table_out"], s["refs_out"] = torch.empty_like(table), torch.empty_like(refs)
    return s


# ------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------
def run(state):
    return (run_own if own else run_plain)[state["case"]["kind"]](state)


def own_rope(s):
    from paper_2609_26100_gb300 import native

    native.qk_rope(s["args"])
    return {"q": s["q_out"], "k": s["k_out"]}


def own_append(s):
    s["cache"].append(0, s["batch"], s["k"], s["v"])
    s["cache"].read(0, s["reads"], s["k_back"], s["v_back"])
    return {"k": s["k_back"], "v": s["v_back"]}


def own_attn(s):
    c = s["case"]
    s["cache"].attention(0, s["batch"], s["q"], s["out"], lse=s["lse"], window=c["window"], sinks=c["sinks"], mask=s["mask"],
                         positions=s["positions"])
    return {"out": s["out"], "lse": s["lse"]}


def own_fork(s):
    s["pages"].free(s["dst"])
    s["pages"].fork(s["src"], s["dst"], s["tokens"])
    return {"pool": s["pool"], "table": s["table"], "held": s["held"], "refs": s["refs"]}


def own_compact(s):
    s["pages"].compact(s["table_out"], s["refs_out"])
    return {"pool": s["pool"], "table": s["table_out"], "refs": s["refs_out"]}


def plain_rope(s):
    c, dtype = s["case"], DTYPES[s["case"]["dtype"]]
    rot = c["rot"]
    cs = s["table"][s["positions"].long()][:, None]
    out = {}
    for name in ("q", "k"):
        x = s[name].float()
        if c["norm"]:
            x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * s[name + "_gain"].float()
        a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if c["inter"] else (x[..., :rot // 2], x[..., rot // 2:rot])
        u, v = a * cs[..., 0] - b * cs[..., 1], b * cs[..., 0] + a * cs[..., 1]
        turned = torch.stack([u, v], -1).flatten(-2) if c["inter"] else torch.cat([u, v], -1)
        out[name] = torch.cat([turned, x[..., rot:]], -1).to(dtype)
    return out


def rows_of(lens, device):
    """For rows of ragged blocks laid end to end: (block of each row, index in its block)."""
    m = torch.tensor(lens, device=device)
    b = torch.repeat_interleave(torch.arange(len(lens), device=device), m)
    return b, torch.arange(len(b), device=device) - (m.cumsum(0) - m)[b]


def quantised(x):
    """Codes (uint8) and parameters of values [..., d]."""
    x = x.float().unflatten(-1, (-1, GROUP))
    z = x.amin(-1).clamp(-65504, 65504).half()
    s = ((x.amax(-1) - z.float()) / 15).clamp(0, 65504).half()
    f = s.float()[..., None]
    c = torch.where(f > 0, (x - z.float()[..., None]) / f, 0.0).round().clamp(0, 15)
    return c.to(torch.uint8).flatten(-2), torch.stack([s, z], -1)


def plain_append(s):
    c = s["case"]
    d, hk, dev = c["d"], c["hk"], s["pool"].device
    blocks = s["pool"].view(s["pool"].shape[0], hk, -1)
    b, i = rows_of(s["n"], dev)
    pos = torch.tensor(s["ctx"], device=dev)[b] + i
    page = s["table"][b, pos // PAGE].long()
    ids, at = torch.unique(page, return_inverse=True)
    kc, vc, kp, vp = (x.clone() for x in unpack(blocks[ids], d))
    for codes, params, x in ((kc, kp, s["k"]), (vc, vp, s["v"])):
        qc, qp = quantised(x)
        codes[at, :, pos % PAGE], params[at, :, pos % PAGE] = qc, qp
    blocks[ids] = pack(kc, vc, kp, vp)
    # and back
    b, i = rows_of(s["look"], dev)
    pos = torch.tensor(s["first"], device=dev)[b] + i
    ids, at = torch.unique(s["table"][b, pos // PAGE].long(), return_inverse=True)
    kc, vc, kp, vp = unpack(blocks[ids], d)
    k, v = (values(codes[at, :, pos % PAGE], params[at, :, pos % PAGE]) for codes, params in ((kc, kp), (vc, vp)))
    return {"k": k.to(s["k"].dtype), "v": v.to(s["v"].dtype)}


def seen(case, ctx, n):
    """Pages that any row of a block sees: (pages of the sinks, first page of the window, pages in all)."""
    total = -(-(ctx + n) // PAGE)
    lo = max(0, ctx - case["window"] + 1) // PAGE if case["window"] else 0
    sink = min(lo, -(-min(case["sinks"], ctx + n) // PAGE)) if case["window"] else 0
    return sink, lo, sink + total - lo


def plain_attn(s):
    c, dev = s["case"], s["pool"].device
    hq, hk, d = c["hq"], c["hk"], c["d"]
    g = hq // hk
    plan = torch.tensor([(x, m, *seen(c, x, m)) for x, m in zip(s["ctx"], s["n"])], device=dev)
    ctx, n, sink, lo, many = plan.unbind(1)
    most, nmax = max(seen(c, x, m)[2] for x, m in zip(s["ctx"], s["n"])), max(s["n"])
    # the pages in sight of each request, the first ones and then the window's
    p = torch.arange(most, device=dev)[None]
    p = torch.where(p < sink[:, None], p, p - sink[:, None] + lo[:, None])
    used = torch.arange(most, device=dev)[None] < many[:, None]
    ids = torch.where(used, s["table"].gather(1, p.clamp(max=s["table"].shape[1] - 1)), 0).long()
    key = (p[..., None] * PAGE + torch.arange(PAGE, device=dev)).flatten(1)  # [B][S] index of each key
    there = used.repeat_interleave(PAGE, 1) & (key < (ctx + n)[:, None])
    kc, vc, kp, vp = unpack(s["pool"].view(s["pool"].shape[0], hk, -1)[ids], d)  # [B][pages][hk][64][...]
    k, v = (values(x, y).transpose(1, 2).reshape(len(plan), hk, -1, d) for x, y in ((kc, kp), (vc, vp)))
    b, i = rows_of(s["n"], dev)
    q = torch.zeros(len(plan), nmax, hq, d, device=dev)
    q[b, i] = s["q"].float()
    q = q.view(len(plan), nmax, hk, g, d).permute(0, 2, 1, 3, 4).reshape(len(plan), hk, nmax * g, d)
    score = (q @ k.transpose(-1, -2)) * d ** -0.5
    # which keys a row sees
    row = torch.arange(nmax, device=dev)
    pos = torch.zeros(len(plan), nmax, dtype=torch.long, device=dev)
    pos[b, i] = s["positions"].long()
    own_row = (key - ctx[:, None]).clamp(0, nmax - 1)
    bits = torch.zeros(len(plan), nmax, nmax, dtype=torch.bool, device=dev)
    if s["mask"] is None:
        bits[:] = row[None, :] <= row[:, None]
    else:
        bits[b, i] = (s["mask"][:, row // 64] >> (row % 64) & 1).bool()
    in_block = key >= ctx[:, None]
    visible = torch.where(in_block[:, None], bits.gather(2, own_row[:, None].expand(-1, nmax, -1)), True) & there[:, None]
    if c["window"]:
        kpos = torch.where(in_block, pos.gather(1, own_row), key)
        near = (pos[:, :, None] - kpos[:, None] < c["window"]) | (key[:, None] < c["sinks"])
        visible = visible & near
    visible = visible[:, None, :, None].expand(-1, hk, -1, g, -1).reshape(len(plan), hk, nmax * g, -1)
    score = torch.where(visible, score, float("-inf"))
    top = score.amax(-1, keepdim=True)
    w = torch.where(visible, (score - torch.where(top > float("-inf"), top, 0.0)).exp(), 0.0)
    total = w.sum(-1, keepdim=True)
    o = (w @ v) / torch.where(total > 0, total, 1.0)
    lse = (top + total.log())[..., 0]
    o = o.view(len(plan), hk, nmax, g, d).permute(0, 2, 1, 3, 4).reshape(len(plan), nmax, hq, d)[b, i]
    lse = lse.view(len(plan), hk, nmax, g).permute(0, 2, 1, 3).reshape(len(plan), nmax, hq)[b, i]
    return {"out": o.to(s["q"].dtype), "lse": lse}


def plain_fork(s):
    table, held, refs, dev = s["table"], s["held"], s["refs"], s["pool"].device
    dst, src, tok = (torch.tensor(s[x], device=dev) for x in ("dst", "src", "tokens"))
    slot = torch.arange(table.shape[1], device=dev)
    # the sequences that are dropped give their pages back
    gone = table[dst]
    refs.index_add_(0, gone.clamp(min=0).flatten().long(), -(slot[None] < held[dst][:, None]).flatten().to(torch.int32))
    table[dst], held[dst] = -1, 0
    # their places take whole pages of the better ones, and a copy of a part-filled last one
    full, tail = tok // PAGE, tok % PAGE > 0
    mine = slot[None] < full[:, None]
    rows = torch.where(mine, table[src], -1)
    refs.index_add_(0, rows.clamp(min=0).flatten().long(), mine.flatten().to(torch.int32))
    free = torch.nonzero(refs == 0)[:, 0][: len(s["dst"])]
    new = free[(tail.cumsum(0) - 1).clamp(min=0)]
    which = torch.nonzero(tail)[:, 0]
    rows[which, full[which]] = new[which].to(torch.int32)
    refs[new[which]] = 1
    s["pool"][:, new[which]] = s["pool"][:, table[src[which], full[which]].long()]
    table[dst], held[dst] = rows, (full + tail).to(torch.int32)
    return {"pool": s["pool"], "table": table, "held": held, "refs": refs}


def plain_compact(s):
    refs, pool = s["refs"], s["pool"]
    used = torch.nonzero(refs > 0)[:, 0]
    n = len(used)
    at = torch.arange(len(refs), device=refs.device)
    old, new = used[used >= n], torch.nonzero((refs == 0) & (at < n))[:, 0]
    at[old] = new
    pool[:, new] = pool[:, old]
    refs_out = torch.zeros_like(refs)
    refs_out[at[used]] = refs[used]
    table = torch.where(s["table"] >= 0, at[s["table"].clamp(min=0).long()].to(torch.int32), -1)
    return {"pool": pool, "table": table, "refs": refs_out}


run_own = {"rope": own_rope, "append": own_append, "attn": own_attn, "fork": own_fork, "compact": own_compact}
run_plain = {"rope": plain_rope, "append": plain_append, "attn": plain_attn, "fork": plain_fork, "compact": plain_compact}


# ------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ------------------------------------------------------------------------------------------------
def work(case):
    kind = case["kind"]
    if kind == "rope":
        n = case["rows"] * (case["hq"] + case["hk"]) * case["d"]
        return {"bytes": 4 * n, "flops": 10 * n}
    if kind == "append":
        rows = sum(ints(case["n"]))
        looks = sum(c + m - max(0, c - case["back"]) for c, m in zip(ints(case["ctx"]), ints(case["n"])))
        token = case["hk"] * case["d"]
        held = case["hk"] * block_bytes(case["d"]) / PAGE
        return {"bytes": (rows + looks) * (4 * token + held), "flops": 10 * rows * token}
    if kind == "attn":
        keys = [sink * PAGE + c + m - lo * PAGE for c, m in zip(ints(case["ctx"]), ints(case["n"])) for sink, lo, _ in [seen(case, c, m)]]
        rows = ints(case["n"])
        return {"bytes": sum(keys) * case["hk"] * block_bytes(case["d"]) / PAGE + sum(rows) * case["hq"] * (4 * case["d"] + 4),
                "flops": sum(4 * r * case["hq"] * k * case["d"] for r, k in zip(rows, keys))}
    if kind == "fork":
        t = ints(case["tokens"])
        mine = [t[i % len(t)] for i in range(case["forks"])]
        tails = sum(x % PAGE > 0 for x in mine)
        return {"bytes": 4 * tails * case["layers"] * case["elems"] + 16 * sum(x // PAGE + 1 for x in mine) + 4 * case["pages"], "flops": 0}
    return {"bytes": 4 * case["moves"] * case["layers"] * case["elems"] + 8 * case["live"] + 8 * case["pages"], "flops": 0}


# ------------------------------------------------------------------------------------------------
# the same in 64 bits
# ------------------------------------------------------------------------------------------------
def exact(case, seed):
    if case["kind"] in ("fork", "compact"):
        return None  # moved values and whole numbers: nothing is computed in floating point
    s = prepare(case, seed)
    return {"rope": exact_rope, "append": exact_append, "attn": exact_attn}[case["kind"]](s)


def exact_rope(s):
    c, out = s["case"], {}
    half = c["rot"] // 2
    i = torch.arange(half, device="cuda")
    first, second = (2 * i, 2 * i + 1) if c["inter"] else (i, i + half)
    t = s["table"].double()[s["positions"].long()]
    turn = torch.complex(t[..., 0], t[..., 1])[:, None]
    for name in ("q", "k"):
        x = s[name].double()
        if c["norm"]:
            x = s[name + "_gain"].double() * x / (x.pow(2).sum(-1, keepdim=True) / c["d"] + 1e-6).sqrt()
        z = torch.complex(x[..., first], x[..., second]) * turn
        y = x.clone()
        y[..., first], y[..., second] = z.real, z.imag
        out[name] = y
    return out


def element(blocks, head, token, d, side):
    """Values in 64 bits of tokens (indices within their pages) from blocks [n][heads][bytes], by the place of each code."""
    x = torch.arange(d, device=blocks.device)[None]
    t = token[:, None]
    g = x // GROUP
    if side == 0:
        code = t * d + (x % GROUP) // 16 * (d // 4) + g * 16 + x % 16
    else:
        h, b, w, i = t // 32, t % 32 // 8, t % 8 // 2, t % 2
        code = PAGE * d + (((h * (d // 4) + x // 4) * 4 + w) * 4 + x % 4) * 8 + b + 4 * i
    mine = blocks[:, head]
    c = mine.gather(1, code // 2).long() >> 4 * (code % 2) & 15
    p = mine[:, PAGE * d:].contiguous().view(torch.float16).double()
    at = (side * PAGE + t) * (d // GROUP) * 2 + 2 * g
    return c.double() * p.gather(1, at) + p.gather(1, at + 1)


def exact_append(s):
    c = s["case"]
    d, hk = c["d"], c["hk"]
    blocks = s["pool"].view(s["pool"].shape[0], hk, -1)
    out = {"k": [], "v": []}
    at = 0
    for b, (ctx, n, first) in enumerate(zip(s["ctx"], s["n"], s["first"])):
        pos = torch.arange(first, ctx, device="cuda")
        pages = s["table"][b, pos // PAGE].long()
        for side, name in enumerate(("k", "v")):
            if len(pos):
                out[name].append(torch.stack([element(blocks[pages], h, pos % PAGE, d, side) for h in range(hk)], 1))
            x = s[name][at:at + n].double().view(n, hk, d // GROUP, GROUP)
            lo, hi = x.min(-1, keepdim=True).values, x.max(-1, keepdim=True).values
            z = lo.half().double()
            step = ((hi - z).float() / 15).half().double()
            code = ((x - z) / torch.where(step > 0, step, 1.0)).round().clamp(0, 15) * (step > 0)
            out[name].append((code * step + z).view(n, hk, d))
        at += n
    return {name: torch.cat(v) for name, v in out.items()}


def exact_attn(s):
    c = s["case"]
    d, hk, g = c["d"], c["hk"], c["hq"] // c["hk"]
    blocks = s["pool"].view(s["pool"].shape[0], hk, -1)
    out, lses, at = [], [], 0
    for b, (ctx, n) in enumerate(zip(s["ctx"], s["n"])):
        pos = s["positions"][at:at + n].long()
        j = torch.arange(ctx + n, device="cuda")
        sets, _ = tree(c, b, n)
        mine = torch.tensor([[x >> i & 1 for i in range(n)] for x in sets], dtype=torch.bool, device="cuda")
        see = torch.cat([torch.ones(n, ctx, dtype=torch.bool, device="cuda"), mine], 1)
        if c["window"]:
            where = torch.cat([j[:ctx], pos])
            see &= (pos[:, None] - where[None] < c["window"]) | (j[None] < c["sinks"])
        keep = see.any(0).nonzero()[:, 0]  # keys that no row sees are left out
        see, pages = see[:, keep], s["table"][b, keep // PAGE].long()
        mine = blocks[pages] if len(pages) * blocks[0].numel() < 1 << 34 else None
        o, lse = torch.empty(n, c["hq"], d, dtype=torch.float64, device="cuda"), torch.empty(n, c["hq"], dtype=torch.float64, device="cuda")
        for h in range(hk):
            rows = blocks[pages, h][:, None] if mine is None else mine[:, h:h + 1]
            k, v = (element(rows, 0, keep % PAGE, d, side) for side in (0, 1))
            score = torch.einsum("ngd,sd->ngs", s["q"][at:at + n, h * g:(h + 1) * g].double(), k) / math.sqrt(d)
            score = score.masked_fill(~see[:, None], float("-inf"))
            lse[:, h * g:(h + 1) * g] = torch.logsumexp(score, -1)
            o[:, h * g:(h + 1) * g] = torch.einsum("ngs,sd->ngd", torch.softmax(score, -1), v)
        out.append(o)
        lses.append(lse)
        at += n
    return {"out": torch.cat(out), "lse": torch.cat(lses)}
