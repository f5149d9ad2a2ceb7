"""Beam search's operators run together, as a decoder would: prompts appended with norms and rotary positions, page rows forked,
then steps of append, attention over the shared prefix, selection and reordering, none of which the host waits for.  A plain model
beside it keeps every beam's rows in lists: at the end the pages hold, bit for bit, what the separate operators append to a cache
of sequences of their own; each step's attention is that of such sequences; each step's choice is the definition's in 64 bits."""
import pytest
import torch

import paged_ref as R
from paper_2609_26100_gb300 import beams, native, paged

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("side_stream", [False, True])
@pytest.mark.parametrize("texts,n,prompts,steps,hq,hk,d,dtype", [
    (1, 4, [200], 5, 8, 2, 128, torch.bfloat16),
    (2, 3, [64, 191], 4, 4, 4, 64, torch.float16),       # a whole page; a tail that fills up
    (3, 8, [1, 63, 300], 3, 8, 1, 128, torch.float16),   # nothing shared at all; 8 rows of a KV head
    (2, 12, [640, 127], 4, 16, 2, 128, torch.bfloat16),  # many rows over shared keys
    (1, 1, [129], 3, 2, 2, 64, torch.bfloat16),          # a single beam
])
def test_search(texts, n, prompts, steps, hq, hk, d, dtype, side_stream):
    rows, vocab, dev = texts * n, 999, "cuda"
    g = torch.Generator(device=dev).manual_seed(7)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=dev).to(dtype)

    table = torch.empty(max(prompts) + steps + 1, d // 2, 2, device=dev)
    freq, factor = native.rope_frequencies(d, 10000.0)
    native.rope_table(freq, table, factor, native.current_stream())
    q_gain, k_gain = 1 + 0.1 * normal(d), 1 + 0.1 * normal(d)
    longest = max(prompts) + steps
    cache = paged.Kv4Cache.allocate(n_layers=1, n_pages=sum(-(-p // 64) for p in prompts) + 4 * rows, n_seqs=rows,
                                    max_pages=-(-longest // 64) + 1, n_q_heads=hq, n_kv_heads=hk, head_dim=d, shared_rows=rows)
    alone = paged.Kv4Cache.allocate(n_layers=1, n_pages=rows * (-(-longest // 64) + 1), n_seqs=rows, max_pages=-(-longest // 64) + 1,
                                    n_q_heads=hq, n_kv_heads=hk, head_dim=d)
    selector = beams.BeamSelector(rows, vocab, n)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream() if side_stream else torch.cuda.current_stream()
    with torch.cuda.stream(stream):
        held = []  # every beam's rows so far: (k before norm and rotation, v)
        for t, p in enumerate(prompts):
            cache.pages.reserve([t * n], [p])
            q, k, v = normal(p, hq, d), normal(p, hk, d), normal(p, hk, d)
            positions = torch.arange(p, dtype=torch.int32, device=dev)
            cache.append_rope(0, cache.batch([t * n], [0], [p]),
                              native.rope_args(q, k, q, None, positions, table, q_gain=q_gain, k_gain=k_gain, to_pages=True), v)
            cache.pages.fork([t * n] * (n - 1), list(range(t * n + 1, t * n + n)), [p] * (n - 1))
            held += [(k, v)] * n
        score = torch.zeros(rows, device=dev)
        done = torch.zeros(rows, dtype=torch.int32, device=dev)
        seqs, seen = list(range(rows)), []
        for step in range(steps):
            length = [p + step for p in prompts for _ in range(n)]
            cache.pages.reserve(seqs, [c + 1 for c in length])
            batch = cache.batch(seqs, length, [1] * rows)
            positions = torch.tensor(length, dtype=torch.int32, device=dev)
            q, k, v = normal(rows, hq, d), normal(rows, hk, d), normal(rows, hk, d)
            raw = k.clone()
            q_out = torch.empty_like(q)
            cache.append_rope(0, batch, native.rope_args(q, k, q_out, None, positions, table, q_gain=q_gain, k_gain=k_gain, to_pages=True), v)
            held = [(torch.cat([a, raw[b:b + 1]]), torch.cat([c, v[b:b + 1]])) for b, (a, c) in enumerate(held)]
            out, plain = torch.empty_like(q_out), torch.empty_like(q_out)
            cache.attention_shared(0, batch, cache.groups([n] * texts, prompts), q_out, out)
            cache.attention(0, batch, q_out, plain)
            logits = normal(rows, vocab)
            score_out = torch.empty(texts, n, device=dev)
            parent, token = (torch.empty(texts, n, dtype=torch.int32, device=dev) for _ in range(2))
            selector.select(logits, score, score_out, parent, token, n_beams=n, done=done, end_token=5)
            cache.pages.reorder(seqs, parent.view(-1), [c + 1 for c in length])
            seen.append((out, plain, q_out, logits, score, done, score_out, parent, token, list(held), length))
            score, done = score_out.view(-1), done[parent.view(-1).long()] | (token.view(-1) == 5).int()
            if step == 0:
                done = done.clone()
                done[rows - 1] = 1  # (one beam ends early)
            order = parent.view(-1).tolist()
            held = [held[i] for i in order]
    stream.synchronize()
    for c in (cache, alone, cache.pages, selector):
        assert c.sync_status() == 0
    # the pages
    final = [p + steps for p in prompts for _ in range(n)]
    alone.pages.reserve(seqs, final)
    for b, (k, v) in enumerate(held):
        rotated = torch.empty_like(k)
        positions = torch.arange(final[b], dtype=torch.int32, device=dev)
        native.qk_rope(native.rope_args(None, k, None, rotated, positions, table, k_gain=k_gain))
        alone.append(0, alone.batch([b], [0], [final[b]]), rotated, v)
    for side in (0, 1):
        for b in range(rows):
            x, y = (R.sequence_values(c.pool[0], c.table, b, final[b], hk, d, side) for c in (cache, alone))
            assert torch.equal(x, y), (side, b)
    assert all(int(r) >= 0 for r in cache.pages.refs) and int(cache.pages.held.sum()) == sum(-(-f // 64) for f in final)
    # attention and choice, step by step
    eps = torch.finfo(dtype).eps
    for out, plain, q, logits, score, done, score_out, parent, token, rows_of, length in seen:
        # both are within half a step of the type and 2^-11 (bf16, weights of one fp16 part) of the same value (values under 8)
        assert float((out.double() - plain.double()).abs().max()) <= 2 * 8 * (eps / 2 + 2.0 ** -11)
        value = logits.double().log_softmax(-1)
        value[done != 0] = -torch.inf
        value[done != 0, 5] = 0.0
        value = (value + score.double()[:, None]).view(texts, n * vocab)
        top = value.topk(n).values
        assert float((top - score_out.double()).abs().max()) <= 2.0 ** -24 * float(top.abs().max()) * 1.01
        at = (parent.long() - torch.arange(texts, device=dev)[:, None] * n) * vocab + token.long()  # (equal values in either order)
        assert torch.equal(value.gather(1, at), top) and all(len(set(x)) == n for x in at.tolist())


@pytest.mark.parametrize("args", [["--beams", "4", "--prompt", "700", "--steps", "4", "--layers", "2"],
                                  ["--beams", "1", "--prompt", "64", "--steps", "2", "--layers", "1"],
                                  ["--beams", "7", "--texts", "3", "--prompt", "1285", "--steps", "5", "--layers", "2", "--vocab", "501"]])
def test_example(args):
    """Attention is compared with a plain fp32 computation on the values read back (bf16 outputs, under 2^-8 of the norm, weights off
    by 2^-12 at most), the values of a step's choice with 64 bits (a float's half step)."""
    from paper_2609_26100_gb300 import longtext
    got = longtext.main(args)
    assert got["error"] < 2.0 ** -8 + 2.0 ** -12
    worst = max(abs(x) for row in got["score"] for x in row)
    assert got["values"] <= 2.0 ** -24 * worst * 1.01
    if got["unshared"] > 100:
        assert got["held"] < got["unshared"]
