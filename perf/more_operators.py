"""Operators of decoding several continuations of one text over the paged 4-bit KV cache: appending keys and
values with their norms and rotary positions on the way, attention of sequences that share a prefix, the choice of
beams over their vocabulary, and the change of places of the beams' pages.

Each is computed twice: in its plain form, elementary torch operations in 32 bits, and (own) by the framework's
kernels through the calls that a program makes.  exact() is the definition in 64 bits.

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
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def listed():
    return [
        # a step of one user's sixteen beams (7B heads), norms on: launches and latency are all there is
        {"name": "append_beams", "kind": "append", "ctx": ",".join(["1031"] * 16), "n": ",".join(["1"] * 16), "hq": 32, "hk": 32,
         "d": 128, "rot": 128, "inter": False, "norm": True, "dtype": "bf16", "factor": 1.0},
        # draft blocks of sixteen long requests (13B heads), part of each head in neighbouring pairs, stretched positions
        {"name": "append_chains", "kind": "append", "ctx": ",".join(str(1000 + 997 * i) for i in range(16)),
         "n": ",".join(["9"] * 16), "hq": 40, "hk": 40, "d": 128, "rot": 64, "inter": True, "norm": False, "dtype": "f16",
         "factor": 8.0},
        # prompts of ragged lengths, some on top of a context (7B heads)
        {"name": "append_prompt", "kind": "append", "ctx": "0,77,512,4095", "n": "4096,2051,1,1023", "hq": 32, "hk": 32,
         "d": 128, "rot": 128, "inter": False, "norm": True, "dtype": "bf16", "factor": 1.0},
        # four beams of a short prompt (7B): latency
        {"name": "shared_few", "kind": "shared", "sizes": "4", "shared": "1024", "extra": 30, "n": 1, "hq": 32, "hk": 32, "d": 128,
         "dtype": "bf16", "window": 0, "sinks": 0, "tree": False},
        # two users' beams over long prompts with ends inside a page, grouped heads
        {"name": "shared_beams", "kind": "shared", "sizes": "16,7", "shared": "8007,15000", "extra": 300, "n": 1, "hq": 32, "hk": 8,
         "d": 128, "dtype": "bf16", "window": 0, "sinks": 0, "tree": False},
        # 64 samples of one long text (7B): many rows over the same keys
        {"name": "shared_samples", "kind": "shared", "sizes": "64", "shared": "32768", "extra": 200, "n": 1, "hq": 32, "hk": 32,
         "d": 128, "dtype": "bf16", "window": 0, "sinks": 0, "tree": False},
        # draft trees of four hypotheses of one text, a window of 4096 and the first tokens
        {"name": "shared_trees", "kind": "shared", "sizes": "4", "shared": "6000", "extra": 700, "n": 33, "hq": 32, "hk": 8,
         "d": 128, "dtype": "f16", "window": 4096, "sinks": 4, "tree": True},
        # one user's four beams over a vocabulary of 32000
        {"name": "select_few", "kind": "select", "groups": 1, "beams": 4, "keep": 4, "vocab": 32000, "dtype": "bf16", "done": 0},
        # eight users, eight beams each, some of them finished, twice as many candidates kept as beams
        {"name": "select_users", "kind": "select", "groups": 8, "beams": 8, "keep": 16, "vocab": 50021, "dtype": "f32", "done": 9},
        # many wide searches over a large vocabulary: the logits' bytes are the cost
        {"name": "select_wide", "kind": "select", "groups": 16, "beams": 32, "keep": 32, "vocab": 131072, "dtype": "bf16", "done": 0},
        # eight beams change places: few pages, a copied tail in every layer
        {"name": "reorder_beams", "kind": "reorder", "layers": 8, "heads": 8, "d": 128, "sizes": "8", "shared": "1000", "extra": 90},
        # sixty-four beams of four long texts in a deep stack
        {"name": "reorder_deep", "kind": "reorder", "layers": 32, "heads": 8, "d": 128, "sizes": "16,16,16,16",
         "shared": "30000,9000,20000,1500", "extra": 700},
    ]


def draw(rng):
    def log_int(lo, hi):
        return min(hi, int(round(lo * (hi / lo) ** rng.random())))

    def texts(values):
        return ",".join(str(v) for v in values)

    kind = rng.choice(("append", "append", "shared", "shared", "shared", "select", "select", "reorder"))
    d = rng.choice((64, 128, 128))
    hk = rng.choice((4, 8, 32, 40))
    hq = hk * (rng.choice((1, 2, 4)) if hk <= 8 else 1)
    dtype = rng.choice(("bf16", "bf16", "f16"))
    if kind == "append":
        b = log_int(1, 32)
        top = max(2, 6000 // b)
        return {"kind": kind, "ctx": texts(rng.randrange(8000) for _ in range(b)), "n": texts(log_int(1, top) for _ in range(b)),
                "hq": hq, "hk": hk, "d": d, "rot": rng.choice((d, d, d // 2)), "inter": rng.random() < 0.4,
                "norm": rng.random() < 0.6, "dtype": dtype, "factor": rng.choice((1.0, 4.0, 8.0))}
    if kind == "shared":
        g = rng.choice((1, 1, 2, 3))
        n = rng.choice((1, 1, 1, 2, 6, 16, 33))
        top = max(2, min(48 // g, 256 // n))
        window = rng.choice((0, 0, 0, log_int(64, 8192)))
        return {"kind": kind, "sizes": texts(log_int(2, top) for _ in range(g)),
                "shared": texts(log_int(64, 24000 if hk <= 8 else 10000) for _ in range(g)), "extra": log_int(1, 1000), "n": n, "hq": hq,
                "hk": hk, "d": d, "dtype": dtype, "window": window, "sinks": rng.choice((0, 4, 70)) if window else 0,
                "tree": n > 4 and rng.random() < 0.5}
    if kind == "select":
        beams = log_int(1, 48)
        groups = log_int(1, max(2, 256 // beams))
        vocab = log_int(2000, 131072)
        return {"kind": kind, "groups": groups, "beams": beams, "keep": min(64, beams * rng.choice((1, 1, 2))), "vocab": vocab,
                "dtype": rng.choice(("bf16", "f16", "f32")), "done": min(groups * (beams - 1), rng.choice((0, 0, 1, groups * beams // 4)))}
    g = rng.choice((1, 2, 4))
    return {"kind": kind, "layers": log_int(1, 24), "heads": rng.choice((4, 8)), "d": d,
            "sizes": texts(log_int(2, 64 // g) for _ in range(g)), "shared": texts(log_int(1, 20000) for _ in range(g)),
            "extra": log_int(1, 700)}


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


def lengths(case):
    """(group, shared tokens, tokens in all) of every sequence of a case whose groups share prefixes."""
    rng = random.Random("%s.%s.%d" % (case["sizes"], case["shared"], case["extra"]))
    return [(g, s, s + rng.randrange(case["extra"] + 1)) for g, (m, s) in enumerate(zip(ints(case["sizes"]), ints(case["shared"])))
            for _ in range(m)]


def shared_tables(seed, seqs, more, spare):
    """Page table of sequences (group, shared, tokens) with room for `more` tokens each, whose whole shared pages are the
    same ones, strewn over a pool with `spare` free pages: (table, pages held by each, pages of the pool)."""
    full = {g: s // PAGE for g, s, _ in seqs}
    need = [-(-(n + more) // PAGE) for _, _, n in seqs]
    total = sum(full.values()) + sum(m - full[g] for m, (g, _, _) in zip(need, seqs))
    ids = permutation(seed, "pages", total + spare).to(torch.int32)
    table = torch.full((len(seqs), max(need) + 1), -1, dtype=torch.int32, device="cuda")
    at, prefix = 0, {}
    for g, m in full.items():
        prefix[g] = ids[at:at + m]
        at += m
    for b, (m, (g, _, _)) in enumerate(zip(need, seqs)):
        table[b, :full[g]] = prefix[g]
        table[b, full[g]:m] = ids[at:at + m - full[g]]
        at += m - full[g]
    return table, need, total + spare


def tree(case, b, n):
    """(ancestor-or-self sets as whole numbers, depths) of request b's block: a chain, or a tree whose every node hangs
    from one of the four before it that came last."""
    rng = random.Random("%s.%d" % (case["shared"], b))
    sets, depth = [], []
    for i in range(n):
        p = max(0, i - 1 - rng.randrange(4)) if case["tree"] and i else i - 1
        sets.append((sets[p] if p >= 0 else 0) | 1 << i)
        depth.append(depth[p] + 1 if p >= 0 else 0)
    return sets, depth


def prepare(case, seed):
    """What a program has in hand before the call."""
    return {"append": prepare_append, "shared": prepare_shared, "select": prepare_select, "reorder": prepare_reorder}[case["kind"]](case, seed)


def prepare_append(case, seed):
    ctx, n, hq, hk, d, rot = ints(case["ctx"]), ints(case["n"]), case["hq"], case["hk"], case["d"], case["rot"]
    dtype, rows = DTYPES[case["dtype"]], sum(n)
    table, _, n_pages = shared_tables(seed, [(b, 0, c + m) for b, (c, m) in enumerate(zip(ctx, n))], 0, 3)
    # the table a model keeps: base 10000, frequencies divided by the factor beyond the first quarter (long waves)
    inv = 10000.0 ** (-torch.arange(rot // 2, dtype=torch.float64, device="cuda") * 2 / rot)
    inv[rot // 8:] /= case["factor"]
    angle = torch.arange(max(c + m for c, m in zip(ctx, n)), dtype=torch.float64, device="cuda")[:, None] * inv
    scale = 0.1 * math.log(case["factor"]) + 1.0
    # q, k and v rows of one projection, without far outliers
    fused = normal(seed, "qkv", (rows, hq + 2 * hk, d)).clamp_(-2.1, 2.1).to(dtype)
    s = {"case": case, "q": fused[:, :hq], "k": fused[:, hq:hq + hk], "v": fused[:, hq + hk:], "ctx": ctx, "n": n, "table": table,
         "pool": filled(seed, n_pages, hk, d), "turns": (torch.stack([angle.cos(), angle.sin()], -1) * scale).float(),
         "positions": torch.cat([torch.arange(c, c + m, device="cuda") for c, m in zip(ctx, n)]).to(torch.int32)}
    for x in ("q", "k"):
        s[x + "_gain"] = (1 + normal(seed, x + "gain", (d,), std=0.05)).to(dtype) if case["norm"] else None
    if own:
        from paper_2609_26100_gb300 import native, paged

        s["cache"] = paged.Kv4Cache(s["pool"][None], table, n_q_heads=hq, n_kv_heads=hk, head_dim=d)
        s["batch"] = s["cache"].batch(list(range(len(ctx))), ctx, n)
        s["q_out"] = torch.empty(rows, hq, d, dtype=dtype, device="cuda")
        s["args"] = native.rope_args(s["q"], s["k"], s["q_out"], None, s["positions"], s["turns"], q_gain=s["q_gain"],
                                     k_gain=s["k_gain"], eps=1e-6, interleaved=case["inter"], to_pages=True)
        s["k_back"], s["v_back"] = (torch.empty(rows, hk, d, dtype=dtype, device="cuda") for _ in range(2))
    return s


def prepare_shared(case, seed):
    seqs, n, hq, d, dtype = lengths(case), case["n"], case["hq"], case["d"], DTYPES[case["dtype"]]
    table, _, n_pages = shared_tables(seed, seqs, n, 3)
    sets = [tree(case, b, n) for b in range(len(seqs))]
    words = [[(x >> 64 * i & (1 << 64) - 1) - (x >> 64 * i + 63 & 1) * (1 << 64) for i in (0, 1)] for a, _ in sets for x in a]
    s = {"case": case, "seqs": seqs, "pool": filled(seed, n_pages, case["hk"], d), "table": table,
         "q": normal(seed, "q", (len(seqs) * n, hq, d), dtype, 2.0),
         "mask": torch.tensor(words, dtype=torch.int64, device="cuda") if case["tree"] else None,
         "positions": torch.tensor([c + x for (_, _, c), (_, dep) in zip(seqs, sets) for x in dep], dtype=torch.int32, device="cuda")}
    if own:
        from paper_2609_26100_gb300 import paged

        s["cache"] = paged.Kv4Cache(s["pool"][None], table, n_q_heads=hq, n_kv_heads=case["hk"], head_dim=d,
                                    shared_rows=len(seqs) * n)
        s["batch"] = s["cache"].batch(list(range(len(seqs))), [c for _, _, c in seqs], [n] * len(seqs))
        s["groups"] = s["cache"].groups(ints(case["sizes"]), ints(case["shared"]))
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(s["q"].shape[:2], dtype=torch.float32, device="cuda")
    return s


def prepare_select(case, seed):
    rows, vocab, keep = case["groups"] * case["beams"], case["vocab"], case["keep"]
    # logits of a decoder: a bell with a few likely tokens
    logits = normal(seed, "logits", (rows, vocab), std=1.6)
    likely = torch.randint(vocab, (rows, 24), generator=generator(seed, "likely"), device="cuda")
    logits.scatter_add_(1, likely, normal(seed, "lift", (rows, 24), std=1.5) + 5.0)
    done = torch.zeros(rows, dtype=torch.int32, device="cuda")
    order = permutation(seed, "done", rows)
    done[order[order % case["beams"] > 0][:case["done"]]] = 1  # (a group's first beam goes on)
    s = {"case": case, "logits": logits.to(DTYPES[case["dtype"]]), "score": normal(seed, "score", (rows,), std=1.5) - 14.0, "done": done}
    if own:
        from paper_2609_26100_gb300 import beams

        s["beams"] = beams.BeamSelector(rows, vocab, keep)
        s["out"] = {"score": torch.empty(case["groups"], keep, device="cuda"),
                    "parent": torch.empty(case["groups"], keep, dtype=torch.int32, device="cuda"),
                    "token": torch.empty(case["groups"], keep, dtype=torch.int32, device="cuda")}
    return s


def prepare_reorder(case, seed):
    seqs, heads, d = lengths(case), case["heads"], case["d"]
    table, need, n_pages = shared_tables(seed, seqs, 0, len(seqs) + 5)
    held = torch.tensor(need, dtype=torch.int32, device="cuda")
    refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    refs.index_add_(0, table[table >= 0].long(), torch.ones_like(table[table >= 0]))
    # half of a group's beams go on, some of them in several places
    rng, parent, at = random.Random(seed), [], 0
    for m in ints(case["sizes"]):
        best = rng.sample(range(m), max(1, m // 2))
        parent += [at + (i if i in best else rng.choice(best)) for i in range(m)]
        at += m
    s = {"case": case, "pool": normal(seed, "pool", (case["layers"], n_pages, heads * block_bytes(d) // 2), torch.bfloat16), "table": table,
         "held": held, "refs": refs, "parent": torch.tensor(parent, dtype=torch.int32, device="cuda"), "tokens": [n for _, _, n in seqs]}
    if own:
        from paper_2609_26100_gb300 import paged

        s["pages"] = paged.PagePool(s["pool"], table, held, refs)
        s["seqs"] = list(range(len(seqs)))
    return s


# ------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------
def run(state):
    return (run_own if own else run_plain)[state["case"]["kind"]](state)


def own_append(s):
    s["cache"].append_rope(0, s["batch"], s["args"], s["v"])
    s["cache"].read(0, s["batch"], s["k_back"], s["v_back"])
    return {"q": s["q_out"], "k": s["k_back"], "v": s["v_back"]}


def own_shared(s):
    c = s["case"]
    s["cache"].attention_shared(0, s["batch"], s["groups"], s["q"], s["out"], lse=s["lse"], window=c["window"], sinks=c["sinks"],
                                mask=s["mask"], positions=s["positions"])
    return {"out": s["out"], "lse": s["lse"]}


def own_select(s):
    c, o = s["case"], s["out"]
    s["beams"].select(s["logits"], s["score"], o["score"], o["parent"], o["token"], n_beams=c["beams"], done=s["done"], end_token=2)
    return o


def own_reorder(s):
    s["pages"].reorder(s["seqs"], s["parent"], s["tokens"])
    return {"pool": s["pool"], "table": s["table"], "held": s["held"], "refs": s["refs"]}


def plain_rope(s, name):
    c = s["case"]
    rot, x = c["rot"], s[name].float()
    cs = s["turns"][s["positions"].long()][:, None]
    if c["norm"]:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * s[name + "_gain"].float()
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if c["inter"] else (x[..., :rot // 2], x[..., rot // 2:rot])
    u, v = a * cs[..., 0] - b * cs[..., 1], b * cs[..., 0] + a * cs[..., 1]
    turned = torch.stack([u, v], -1).flatten(-2) if c["inter"] else torch.cat([u, v], -1)
    return torch.cat([turned, x[..., rot:]], -1).to(s[name].dtype)


def rows_of(lens, device):
    """For rows of ragged blocks laid end to end: (block of each row, index in its block)."""
    m = torch.tensor(lens, device=device)
    b = torch.repeat_interleave(torch.arange(len(lens), device=device), m)
    return b, torch.arange(len(b), device=device) - (m.cumsum(0) - m)[b]


def quantised(x):
    """Codes (uint8) and parameters of values [..., d]."""
    x = x.float().unflatten(-1, (-1, GROUP))
    z = x.amin(-1).clamp(-65504, 65504).half()
    s = ((x.amax(-1) - z.float()) / torch.full((), 15.0, device=x.device)).clamp(0, 65504).half()
    f = s.float()[..., None]
    c = torch.where(f > 0, (x - z.float()[..., None]) / f, 0.0).round().clamp(0, 15)
    return c.to(torch.uint8).flatten(-2), torch.stack([s, z], -1)


def plain_append(s):
    c = s["case"]
    d, dev = c["d"], s["pool"].device
    q, k = plain_rope(s, "q"), plain_rope(s, "k")
    blocks = s["pool"].view(s["pool"].shape[0], c["hk"], -1)
    b, i = rows_of(s["n"], dev)
    pos = torch.tensor(s["ctx"], device=dev)[b] + i
    ids, at = torch.unique(s["table"][b, pos // PAGE].long(), return_inverse=True)
    kc, vc, kp, vp = (x.clone() for x in unpack(blocks[ids], d))
    kc[at, :, pos % PAGE], kp[at, :, pos % PAGE] = quantised(k)
    vc[at, :, pos % PAGE], vp[at, :, pos % PAGE] = quantised(s["v"])
    blocks[ids] = pack(kc, vc, kp, vp)
    # and back
    kc, vc, kp, vp = unpack(blocks[ids], d)
    k, v = (values(codes[at, :, pos % PAGE], params[at, :, pos % PAGE]) for codes, params in ((kc, kp), (vc, vp)))
    return {"q": q, "k": k.to(s["k"].dtype), "v": v.to(s["v"].dtype)}


def scores_of(q, blocks, d):
    """Scores of rows q [n][heads][rows][d] with the keys of pages blocks [n][pages][heads][bytes], and the values."""
    kc, vc, kp, vp = unpack(blocks, d)
    k, v = (values(x, y).transpose(1, 2).flatten(2, 3) for x, y in ((kc, kp), (vc, vp)))
    return (q @ k.transpose(-1, -2)) * d ** -0.5, v


def plain_shared(s):
    c, dev, seqs = s["case"], s["pool"].device, s["seqs"]
    hq, hk, d, n, sizes = c["hq"], c["hk"], c["d"], c["n"], ints(c["sizes"])
    g, blocks = hq // hk, s["pool"].view(s["pool"].shape[0], c["hk"], -1)
    group, member = rows_of(sizes, dev)
    ctx = torch.tensor([x for _, _, x in seqs], device=dev)
    full = torch.tensor([x // PAGE for x in ints(c["shared"])], device=dev)
    pos = s["positions"].long().view(-1, n)

    def softmax_parts(score, v, seen):
        score = torch.where(seen, score, float("-inf"))
        top = score.amax(-1, keepdim=True)
        w = torch.where(seen, (score - torch.where(top > float("-inf"), top, 0.0)).exp(), 0.0)
        return top[..., 0], w.sum(-1), w @ v

    q = s["q"].float().view(-1, n, hk, g, d).transpose(1, 2)  # [sequence][kv head][row][head][d]
    # the shared pages, once a group: its sequences' rows side by side
    pages = torch.arange(int(full.max()), device=dev)
    first = torch.tensor([sum(sizes[:i]) for i in range(len(sizes))], device=dev)
    ids = torch.where(pages < full[:, None], s["table"][first][:, :len(pages)], 0).long()
    rows = torch.zeros(len(sizes), max(sizes), hk, n, g, d, device=dev)
    rows[group, member] = q
    at = torch.zeros(len(sizes), max(sizes), n, dtype=torch.long, device=dev)
    at[group, member] = pos
    key = torch.arange(len(pages) * PAGE, device=dev)
    score, v = scores_of(rows.transpose(1, 2).flatten(2, 4), blocks[ids], d)
    seen = (key < full[:, None] * PAGE)[:, None]
    if c["window"]:
        seen = seen & ((at.flatten(1)[..., None] - key < c["window"]) | (key < c["sinks"]))
    seen = seen.expand(-1, max(sizes) * n, -1).repeat_interleave(g, 1)[:, None]
    parts = [x.unflatten(2, (max(sizes), n, g)).transpose(1, 2)[group, member] for x in softmax_parts(score, v, seen)]
    # every sequence's own pages
    mine = full[group]
    many = -(-(ctx + n) // PAGE) - mine
    pages = torch.arange(int(many.max()), device=dev)
    where = (mine[:, None] + pages).clamp(max=s["table"].shape[1] - 1)
    ids = torch.where(pages < many[:, None], s["table"].gather(1, where), 0).long()
    key = mine[:, None] * PAGE + torch.arange(len(pages) * PAGE, device=dev)
    score, v = scores_of(q.flatten(2, 3), blocks[ids], d)
    slot = (key - ctx[:, None]).clamp(0, n - 1)
    row = torch.arange(n, device=dev)
    bits = row[None, :] <= row[:, None] if s["mask"] is None else ((s["mask"][:, row // 64] >> (row % 64)) & 1).bool()
    bits = bits.expand(len(seqs), n, n) if s["mask"] is None else bits.view(-1, n, n)
    fresh = key >= ctx[:, None]
    seen = torch.where(fresh[:, None], bits.gather(2, slot[:, None].expand(-1, n, -1)), True) & (key < ctx[:, None] + n)[:, None]
    if c["window"]:
        kpos = torch.where(fresh, pos.gather(1, slot), key)
        seen = seen & ((pos[:, :, None] - kpos[:, None] < c["window"]) | (key[:, None] < c["sinks"]))
    parts2 = [x.unflatten(2, (n, g)) for x in softmax_parts(score, v, seen.repeat_interleave(g, 1)[:, None])]
    # and both together
    top = torch.maximum(parts[0], parts2[0])
    base = torch.where(top > float("-inf"), top, 0.0)
    a, b = (parts[0] - base).exp(), (parts2[0] - base).exp()
    total = a * parts[1] + b * parts2[1]
    o = (a[..., None] * parts[2] + b[..., None] * parts2[2]) / torch.where(total > 0, total, 1.0)[..., None]
    return {"out": o.transpose(1, 2).reshape(-1, hq, d).to(s["q"].dtype), "lse": (top + total.log()).transpose(1, 2).reshape(-1, hq)}


def plain_select(s):
    c = s["case"]
    # in 64 bits: which of two candidates is larger goes by their last bits
    x = s["logits"].double()
    top = x.amax(-1, keepdim=True)
    value = s["score"].double()[:, None] + (x - (top + (x - top).exp().sum(-1, keepdim=True).log()))
    token = torch.arange(c["vocab"], device=x.device)
    value = torch.where(s["done"][:, None] > 0, torch.where(token == 2, s["score"].double()[:, None], float("-inf")), value)
    best, at = torch.sort(value.view(c["groups"], -1), dim=-1, descending=True, stable=True)
    best, at = best[:, :c["keep"]], at[:, :c["keep"]]
    base = torch.arange(c["groups"], device=x.device)[:, None] * c["beams"]
    return {"score": best.float(), "parent": (base + at // c["vocab"]).to(torch.int32), "token": (at % c["vocab"]).to(torch.int32)}


def plain_reorder(s):
    table, held, refs, dev = s["table"], s["held"], s["refs"], s["pool"].device
    n, slot = table.shape[0], torch.arange(table.shape[1], device=dev)
    parent, tokens = s["parent"].long(), torch.tensor(s["tokens"], device=dev)
    # the place that keeps a beam's part-filled last page: its own if it goes on there, else the lowest
    me = torch.arange(n, device=dev)
    child = parent[None, :] == me[:, None]
    keeper = torch.where(parent == me, me, child.to(torch.uint8).argmax(1))
    full, tail = (tokens // PAGE)[parent], (tokens % PAGE > 0)[parent]
    copied = tail & (keeper[parent] != me)
    rows = torch.where(slot < (full + tail)[:, None], table[parent], -1)
    source = rows.gather(1, full.clamp(max=table.shape[1] - 1)[:, None])[:, 0]
    free = torch.nonzero(refs == 0)[:, 0][:n]
    new = free[(copied.cumsum(0) - 1).clamp(min=0)].to(torch.int32)
    which = torch.nonzero(copied)[:, 0]
    rows[which, full[which]] = new[which]
    # what each page is held by
    refs.index_add_(0, table.clamp(min=0).flatten().long(), -(slot < held[:, None]).flatten().to(torch.int32))
    refs.index_add_(0, rows.clamp(min=0).flatten().long(), (slot < (full + tail)[:, None]).flatten().to(torch.int32))
    s["pool"][:, new[which].long()] = s["pool"][:, source[which].long()]
    table.copy_(rows)
    held.copy_(full + tail)
    return {"pool": s["pool"], "table": table, "held": held, "refs": refs}


run_own = {"append": own_append, "shared": own_shared, "select": own_select, "reorder": own_reorder}
run_plain = {"append": plain_append, "shared": plain_shared, "select": plain_select, "reorder": plain_reorder}


# ------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ------------------------------------------------------------------------------------------------
def in_sight(case, first, ctx, end):
    """Tokens of [first, end) in pages of which a row at ctx or later sees some: those of the first tokens and of the window."""
    if not case["window"]:
        return end - first
    lo = min(end, max(first, max(0, ctx - case["window"] + 1) // PAGE * PAGE))
    sink = max(0, min(lo, -(-case["sinks"] // PAGE) * PAGE) - first)
    return end - lo + sink


def work(case):
    kind = case["kind"]
    held = lambda d: block_bytes(d) / PAGE  # noqa: E731
    if kind == "append":
        rows, width = sum(ints(case["n"])), 2
        # (rows read, q and the values read back written, pages written and read, a row of the rotations' table each)
        return {"bytes": rows * (width * case["d"] * (2 * case["hq"] + 4 * case["hk"]) + 2 * case["hk"] * held(case["d"]) + 4 * case["rot"]),
                "flops": 10 * rows * (case["hq"] + 2 * case["hk"]) * case["d"]}
    if kind == "shared":
        seqs, n = lengths(case), case["n"]
        keys = flops = 0
        for g, (m, sh) in enumerate(zip(ints(case["sizes"]), ints(case["shared"]))):
            base = sh // PAGE * PAGE
            ctx = [c for x, _, c in seqs if x == g]
            one = in_sight(case, 0, min(ctx), base)
            mine = [in_sight(case, base, c, c + n) for c in ctx]
            keys += one + sum(mine)
            flops += sum(4 * n * case["hq"] * (one + x) * case["d"] for x in mine)
        return {"bytes": keys * case["hk"] * held(case["d"]) + len(seqs) * n * case["hq"] * (4 * case["d"] + 4), "flops": flops}
    if kind == "select":
        rows = case["groups"] * case["beams"] - case["done"]
        return {"bytes": rows * case["vocab"] * (4 if case["dtype"] == "f32" else 2) + case["groups"] * case["keep"] * 12,
                "flops": 3 * rows * case["vocab"]}
    seqs, at, copies, sizes = lengths(case), 0, 0, ints(case["sizes"])
    for m in sizes:  # at most m - m // 2 places take another's beam, each with a tail
        copies += sum(sorted((c % PAGE > 0 for _, _, c in seqs[at:at + m]))[:m - max(1, m // 2)])
        at += m
    page = case["heads"] * block_bytes(case["d"])
    return {"bytes": 2 * copies * case["layers"] * page + 8 * sum(-(-c // PAGE) for _, _, c in seqs), "flops": 0}


# ------------------------------------------------------------------------------------------------
# the same in 64 bits
# ------------------------------------------------------------------------------------------------
def exact(case, seed):
    if case["kind"] == "reorder":
        return None  # moved values and whole numbers: nothing is computed in floating point
    s = prepare(case, seed)
    return {"append": exact_append, "shared": exact_shared, "select": exact_select}[case["kind"]](s)


def exact_append(s):
    c, out = s["case"], {}
    d, half = c["d"], c["rot"] // 2
    i = torch.arange(half, device="cuda")
    first, second = (2 * i, 2 * i + 1) if c["inter"] else (i, i + half)
    t = s["turns"].double()[s["positions"].long()]
    turn = torch.complex(t[..., 0], t[..., 1])[:, None]
    for name in ("q", "k"):
        x = s[name].double()
        if c["norm"]:
            x = s[name + "_gain"].double() * x / (x.pow(2).sum(-1, keepdim=True) / d + 1e-6).sqrt()
        z = torch.complex(x[..., first], x[..., second]) * turn
        y = x.clone()
        y[..., first], y[..., second] = z.real, z.imag
        out[name] = y
    for name, x in (("k", out["k"].to(s["k"].dtype)), ("v", s["v"])):
        x = x.double().reshape(-1, c["hk"], d // GROUP, GROUP)
        lo, hi = x.min(-1, keepdim=True).values, x.max(-1, keepdim=True).values
        z = lo.half().double()
        step = ((hi - z) / 15).half().double()
        code = ((x - z) / torch.where(step > 0, step, 1.0)).round().clamp(0, 15) * (step > 0)
        out[name] = (code * step + z).view(-1, c["hk"], d)
    return out


def element(blocks, token, d, side):
    """Values in 64 bits of tokens (indices within their pages) from one head's blocks [n][bytes], by the place of each code."""
    x = torch.arange(d, device=blocks.device)[None]
    t = token[:, None]
    g = x // GROUP
    if side == 0:
        code = t * d + (x % GROUP) // 16 * (d // 4) + g * 16 + x % 16
    else:
        h, b, w, i = t // 32, t % 32 // 8, t % 8 // 2, t % 2
        code = PAGE * d + (((h * (d // 4) + x // 4) * 4 + w) * 4 + x % 4) * 8 + b + 4 * i
    c = blocks.gather(1, code // 2).long() >> 4 * (code % 2) & 15
    p = blocks[:, PAGE * d:].contiguous().view(torch.float16).double()
    at = (side * PAGE + t) * (d // GROUP) * 2 + 2 * g
    return c.double() * p.gather(1, at) + p.gather(1, at + 1)


def exact_shared(s):
    c, seqs = s["case"], s["seqs"]
    d, hk, g, n = c["d"], c["hk"], c["hq"] // c["hk"], c["n"]
    blocks = s["pool"].view(s["pool"].shape[0], hk, -1)
    out = torch.empty(len(seqs) * n, c["hq"], d, dtype=torch.float64, device="cuda")
    lse = torch.empty(len(seqs) * n, c["hq"], dtype=torch.float64, device="cuda")
    for h in range(hk):
        common = {}
        for b, (group, shared, ctx) in enumerate(seqs):
            base, rows = shared // PAGE * PAGE, slice(b * n, (b + 1) * n)
            j = torch.arange(ctx + n, device="cuda")
            pages = s["table"][b, j // PAGE].long()
            if group not in common:
                common[group] = [element(blocks[pages[:base], h], j[:base] % PAGE, d, side) for side in (0, 1)]
            k, v = (torch.cat([common[group][side], element(blocks[pages[base:], h], j[base:] % PAGE, d, side)]) for side in (0, 1))
            pos = s["positions"][rows].long()
            sets, _ = tree(c, b, n)
            mine = torch.tensor([[x >> i & 1 for i in range(n)] for x in sets], dtype=torch.bool, device="cuda")
            see = torch.cat([torch.ones(n, ctx, dtype=torch.bool, device="cuda"), mine], 1)
            if c["window"]:
                see &= (pos[:, None] - torch.cat([j[:ctx], pos])[None] < c["window"]) | (j[None] < c["sinks"])
            score = torch.einsum("ngd,sd->ngs", s["q"][rows, h * g:(h + 1) * g].double(), k) / math.sqrt(d)
            score = score.masked_fill(~see[:, None], float("-inf"))
            lse[rows, h * g:(h + 1) * g] = torch.logsumexp(score, -1)
            out[rows, h * g:(h + 1) * g] = torch.einsum("ngs,sd->ngd", torch.softmax(score, -1), v)
    return {"out": out, "lse": lse}


def exact_select(s):
    c = s["case"]
    lse = torch.logsumexp(s["logits"].double(), -1)
    score = s["score"].double()
    # a row's n-th largest logit: the candidates that a group chooses from
    k = min(c["keep"], c["vocab"])
    value = torch.topk(s["logits"].double(), k, -1).values + (score - lse)[:, None]
    value[s["done"] > 0] = float("-inf")
    value[s["done"] > 0, 0] = score[s["done"] > 0]
    return {"score": torch.topk(value.view(c["groups"], -1), c["keep"], -1).values, "parent": None, "token": None}
