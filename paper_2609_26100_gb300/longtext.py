"""Example: several continuations of one long prompt over a paged 4-bit KV cache.

    python -m paper_2609_26100_gb300.longtext [--prompt 3000] [--steps 6] [--hypotheses 4] [--layers 4]
    python -m paper_2609_26100_gb300.longtext --beams 8 [--texts 2] [--prompt 3000] [--steps 6] [--layers 4]

A stack of attention layers with random weights (head norms, rotary positions stretched for a long
context, grouped heads; every second layer sees a window and the first tokens) decodes speculatively:

  * the prompt enters in chunks of 128 rows: project, norm and rotate (tss_qk_rope), append
    (tss_paged_append), attend (tss_paged_attention);
  * its pages are shared by all hypotheses (tss_pages_fork), a part-filled last page is copied;
  * a step scores a draft tree for every hypothesis, takes a path of it, and appends the path's rows in
    order over the block's; pages past it are given back (tss_pages_free);
  * every second step the worse half is dropped and forked from the better half; at the end the pool is
    made dense (tss_pages_compact).

With --beams it searches instead: every text's beams share its prompt's pages; a step norms, rotates and appends in
one launch (tss_paged_append_rope), attends with the shared keys read once (tss_paged_attention_shared), picks the
best continuations over beams and vocabulary (tss_beam_select) and lets page rows follow their parents
(tss_pages_reorder), all without a host wait.

It checks the attention against a plain computation on the values read back (tss_paged_read) and prints the
error and the time of a step.
"""
from __future__ import annotations

import argparse
import random
import time

import torch

from . import beams, native, paged

WINDOW, SINKS = 512, 4


class Stack:
    def __init__(self, layers: int, n_q_heads: int, n_kv_heads: int, head_dim: int, max_positions: int, seed: int):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.layers, self.hq, self.hk, self.d = layers, n_q_heads, n_kv_heads, head_dim
        self.width = n_q_heads * head_dim

        def matrix(rows, cols):
            return (torch.randn(rows, cols, generator=g, device="cuda") * cols ** -0.5).bfloat16()

        self.wqkv = [matrix(self.width + 2 * n_kv_heads * head_dim, self.width) for _ in range(layers)]
        self.wo = [matrix(self.width, self.width) for _ in range(layers)]
        self.gains = [(1 + 0.2 * torch.randn(2, head_dim, generator=g, device="cuda")).bfloat16() for _ in range(layers)]
        freq, factor = native.rope_frequencies(head_dim, 10000.0, "yarn", max(1.0, max_positions / 2048), 2048.0)
        self.table = torch.empty(max_positions, head_dim // 2, 2, device="cuda")
        native.rope_table(freq, self.table, factor, native.current_stream())
        self.error = 0.0

    def run(self, cache: paged.Kv4Cache, batch, x, positions, mask=None, check=None, joined=False, groups=None):
        """Rows x of the batch's blocks through all layers, their keys and values appended on the way; the
        outputs and each layer's keys (rotated, unless joined) and values.  check: a request whose first layer is compared
        with a plain computation; joined: rotated and appended in one launch; groups: requests that share pages."""
        kept = []
        for layer in range(self.layers):
            n = x.shape[0]
            rows = torch.nn.functional.linear(x / x.float().square().mean(-1, keepdim=True).sqrt().bfloat16(), self.wqkv[layer])
            rows = rows.view(n, self.hq + 2 * self.hk, self.d)
            q, k, v = rows[:, :self.hq], rows[:, self.hq:self.hq + self.hk], rows[:, self.hq + self.hk:]
            args = native.rope_args(q, k, q, None if joined else k, positions, self.table, q_gain=self.gains[layer][0],
                                    k_gain=self.gains[layer][1], to_pages=joined)
            if joined:
                cache.append_rope(layer, batch, args, v)
            else:
                native.qk_rope(args)
                cache.append(layer, batch, k, v)
            out = torch.empty(n, self.hq, self.d, dtype=x.dtype, device=x.device)
            near = {"window": WINDOW, "sinks": SINKS} if layer % 2 else {}
            if groups is not None:
                cache.attention_shared(layer, batch, groups, q, out, mask=mask, positions=positions, **near)
            else:
                cache.attention(layer, batch, q, out, mask=mask, positions=positions, **near)
            if check is not None and layer < 2:
                self.compare(cache, layer, check, q, out, near)
            x = x + torch.nn.functional.linear(out.view(n, -1), self.wo[layer])
            kept.append((k, v))
        return x, kept

    def compare(self, cache, layer, check, q, out, near):
        """check: (sequence, first, rows, offset in q, ancestor sets, positions) of one request."""
        seq, first, n, at, sets, pos = check
        k, v = (torch.empty(first + n, self.hk, self.d, device="cuda") for _ in range(2))
        cache.read(layer, cache.batch([seq], [0], [first + n]), k, v)
        g = self.hq // self.hk
        see = torch.ones(n, first + n, dtype=torch.bool)
        see[:, first:] = torch.tensor([[s >> i & 1 for i in range(n)] for s in sets], dtype=torch.bool)
        if near:
            where = torch.cat([torch.arange(first), torch.tensor(pos)])
            see &= (torch.tensor(pos)[:, None] - where[None] < WINDOW) | (torch.arange(first + n)[None] < SINKS)
        score = torch.einsum("nhd,shd->hns", q[at:at + n].float(), k.repeat_interleave(g, 1)) * self.d ** -0.5
        weight = score.masked_fill(~see.cuda()[None], float("-inf")).softmax(-1)
        ref = torch.einsum("hns,shd->nhd", weight, v.repeat_interleave(g, 1))
        self.error = max(self.error, float((out[at:at + n].float() - ref).norm() / ref.norm()))


def draft_tree(rng: random.Random, nodes: int):
    """Parents of a random draft tree under its root: (ancestor-or-self sets, depths, parents)."""
    parents = [-1] + [rng.randrange(max(0, i - 4), i) for i in range(1, nodes)]
    sets, depth = [], []
    for i, p in enumerate(parents):
        sets.append((sets[p] if p >= 0 else 0) | 1 << i)
        depth.append(depth[p] + 1 if p >= 0 else 0)
    return sets, depth, parents


def mask_words(sets):
    signed = lambda x: x - (1 << 64) if x >> 63 else x  # noqa: E731
    return [[signed(s & (1 << 64) - 1), signed(s >> 64)] for s in sets]


def search(a) -> dict:
    """Beam search of a.texts texts, a.beams beams each; end token 0."""
    texts, n, rows = a.texts, a.beams, a.texts * a.beams
    prompts = [max(1, a.prompt - 100 * i) for i in range(texts)]
    stack, pages = Stack(a.layers, 16, 4, 128, a.prompt + a.steps + 1, a.seed), paged.PAGE_TOKENS
    # (while rows change places a text's beams hold at most what they held, and a tail and a new page each)
    cache = paged.Kv4Cache.allocate(n_layers=a.layers, n_pages=sum(-(-p // pages) for p in prompts) + rows * (3 + a.steps // pages),
                                    n_seqs=rows, max_pages=-(-(a.prompt + a.steps + 1) // pages) + 1, n_q_heads=16, n_kv_heads=4,
                                    head_dim=128, shared_rows=rows)
    g = torch.Generator(device="cuda").manual_seed(a.seed)
    head, embed = ((torch.randn(a.vocab, stack.width, generator=g, device="cuda") * w).bfloat16() for w in (4 * stack.width ** -0.5, 1.0))
    first, step_of = beams.BeamSelector(texts, a.vocab, n), beams.BeamSelector(rows, a.vocab, n)

    def normal(x):
        return x / x.float().square().mean(-1, keepdim=True).sqrt().bfloat16()

    # the prompts, each in the row of its text's first beam
    ends = []
    for t, prompt in enumerate(prompts):
        x = torch.randn(prompt, stack.width, generator=g, device="cuda").bfloat16()
        cache.pages.reserve([t * n], [prompt])
        for at in range(0, prompt, 128):
            m = min(128, prompt - at)
            positions = torch.arange(at, at + m, dtype=torch.int32, device="cuda")
            check = (t * n, at, m, 0, [(2 << i) - 1 for i in range(m)], list(range(at, at + m)))
            last, _ = stack.run(cache, cache.batch([t * n], [at], [m]), x[at:at + m], positions, check=check, joined=True)
        ends.append(last[-1])
        cache.pages.fork([t * n] * (n - 1), [t * n + i for i in range(1, n)], [prompt] * (n - 1))

    def chosen(selector, logits, was, done, width):
        """A step's choice, compared with a plain one of the same logits."""
        out = torch.empty(texts, n, device="cuda"), *(torch.empty(texts, n, dtype=torch.int32, device="cuda") for _ in range(2))
        selector.select(logits, was, *out, n_beams=width, done=done, end_token=0)
        return out

    def off(logits, was, done, width, score):
        value = logits.double().log_softmax(-1)
        if done is not None:  # (finished beams go on with the end token, at no cost)
            value[done != 0] = -torch.inf
            value[done != 0, 0] = 0.0
        value = (value if was is None else value + was.double()[:, None]).view(texts, width * a.vocab)
        return float((value.topk(n).values - score.double()).abs().max())

    logits = torch.nn.functional.linear(normal(torch.stack(ends)), head)
    score, _, token = chosen(first, logits, None, None, 1)
    error, taken = off(logits, None, None, 1, score), 0.0
    done = (token.view(-1) == 0).int()
    parents, tokens, seqs = [], [token.view(-1)], list(range(rows))
    for step in range(a.steps):
        length = [p + step for p in prompts for _ in range(n)]
        torch.cuda.synchronize()
        began = time.perf_counter()
        cache.pages.reserve(seqs, [c + 1 for c in length])
        positions = torch.tensor(length, dtype=torch.int32, device="cuda")
        check = (rows - 1, length[-1], 1, rows - 1, [1], [length[-1]]) if step % 2 else None
        out, _ = stack.run(cache, cache.batch(seqs, length, [1] * rows), embed[tokens[-1].long()], positions, check=check, joined=True,
                           groups=cache.groups([n] * texts, prompts))
        logits, was, over = torch.nn.functional.linear(normal(out), head), score.view(-1), done
        score, parent, token = chosen(step_of, logits, was, over, n)
        cache.pages.reorder(seqs, parent.view(-1), [c + 1 for c in length])
        parents.append(parent.view(-1))
        tokens.append(token.view(-1))
        done = done[parent.view(-1).long()] | (token.view(-1) == 0).int()
        torch.cuda.synchronize()
        taken += time.perf_counter() - began
        error = max(error, off(logits, was, over, n, score))
    held = int((cache.pages.refs > 0).sum())
    for status in (cache.sync_status(), cache.pages.sync_status(), first.sync_status(), step_of.sync_status()):
        native.check(status, "longtext")
    # every beam's tokens, from its last one back
    row, found = torch.arange(rows, device="cuda"), [tokens[-1]]
    for parent, token in zip(reversed(parents), reversed(tokens[:-1])):
        row = parent[row].long()
        found.append(token[row])
    found = torch.stack(found[::-1], 1).view(texts, n, -1).tolist()
    full = sum(n * -(-(p + a.steps) // pages) for p in prompts)
    print(f"{texts} x {n} beams, best {score[0, 0].item():.2f} with {found[0][0][:8]}, {held} pages ({full} unshared), "
          f"{taken / max(a.steps, 1) * 1e3:.2f} ms a step, attention off by {stack.error:.1e}, values by {error:.1e}")
    cache.close()
    return {"error": stack.error, "held": held, "unshared": full, "values": error, "score": score.tolist(), "tokens": found}


def main(argv=None) -> dict:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--prompt", type=int, default=3000)
    ap.add_argument("--steps", type=int, default=6)
    ap.add_argument("--hypotheses", type=int, default=4)
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--nodes", type=int, default=12, help="rows of a draft tree, its root included")
    ap.add_argument("--seed", type=int, default=1)
    ap.add_argument("--beams", type=int, default=0, help="beams of a text; 0: draft trees instead")
    ap.add_argument("--texts", type=int, default=1, help="texts that are searched together")
    ap.add_argument("--vocab", type=int, default=8000)
    a = ap.parse_args(argv)
    if a.beams:
        return search(a)
    rng = random.Random(a.seed)
    n, longest = a.hypotheses, a.prompt + a.steps * a.nodes + a.nodes
    stack = Stack(a.layers, 16, 4, 128, longest, a.seed)
    pages = paged.PAGE_TOKENS
    cache = paged.Kv4Cache.allocate(n_layers=a.layers, n_pages=-(-a.prompt // pages) + 2 * n * (2 + a.steps * a.nodes // pages),
                                    n_seqs=n, max_pages=-(-longest // pages) + 1, n_q_heads=16, n_kv_heads=4, head_dim=128)

    # the prompt, in sequence 0
    x = torch.randn(a.prompt, stack.width, generator=torch.Generator(device="cuda").manual_seed(a.seed), device="cuda").bfloat16()
    cache.pages.reserve([0], [a.prompt])
    for first in range(0, a.prompt, 128):
        m = min(128, a.prompt - first)
        positions = torch.arange(first, first + m, dtype=torch.int32, device="cuda")
        check = (0, first, m, 0, [(2 << i) - 1 for i in range(m)], list(range(first, first + m)))
        last, _ = stack.run(cache, cache.batch([0], [first], [m]), x[first:first + m], positions, check=check)
    cache.pages.fork([0] * (n - 1), list(range(1, n)), [a.prompt] * (n - 1))

    length, total = [a.prompt] * n, torch.zeros(n)
    state = last[-1:].repeat(n, 1)
    taken = 0.0
    for step in range(a.steps):
        trees = [draft_tree(rng, a.nodes) for _ in range(n)]
        cache.pages.reserve(list(range(n)), [c + a.nodes for c in length])
        batch = cache.batch(list(range(n)), length, [a.nodes] * n)
        pos = [[c + d for d in t[1]] for c, t in zip(length, trees)]
        positions = torch.tensor([p for row in pos for p in row], dtype=torch.int32, device="cuda")
        mask = torch.tensor([w for t in trees for w in mask_words(t[0])], dtype=torch.int64, device="cuda")
        rows = state.repeat_interleave(a.nodes, 0) + 0.3 * torch.randn(
            n * a.nodes, stack.width, device="cuda", generator=torch.Generator(device="cuda").manual_seed(100 + step)).bfloat16()
        check = (n - 1, length[n - 1], a.nodes, (n - 1) * a.nodes, trees[n - 1][0], pos[n - 1])
        torch.cuda.synchronize()
        began = time.perf_counter()
        out, kept = stack.run(cache, batch, rows, positions, mask, check=check if step % 2 else None)
        # a path of each tree is accepted: its rows, in order, take the block's place in the cache
        score = out.float().square().mean(-1).view(n, a.nodes).cpu()
        paths = []
        for b, (_, _, parents) in enumerate(trees):
            leaf, path = max(range(a.nodes), key=lambda i: float(score[b, i])), []
            while leaf >= 0:
                path, leaf = [leaf] + path, parents[leaf]
            paths.append(path)
        index = torch.tensor([b * a.nodes + i for b, p in enumerate(paths) for i in p], device="cuda")
        again = cache.batch(list(range(n)), length, [len(p) for p in paths])
        for layer, (k, v) in enumerate(kept):
            cache.append(layer, again, k[index], v[index])
        length = [c + len(p) for c, p in zip(length, paths)]
        cache.pages.free(list(range(n)), length)
        state = torch.stack([out[b * a.nodes + p[-1]] for b, p in enumerate(paths)])
        total += torch.tensor([float(score[b, p[-1]]) for b, p in enumerate(paths)])
        if step % 2 and n > 1:  # the better half goes on twice
            order = sorted(range(n), key=lambda b: -float(total[b]))
            best, worst = order[:n // 2], order[n - n // 2:]
            cache.pages.free(worst)
            cache.pages.fork(best, worst, [length[b] for b in best])
            for b, w in zip(best, worst):
                length[w], total[w], state[w] = length[b], total[b], state[b]
        torch.cuda.synchronize()
        taken += time.perf_counter() - began
    held = int((cache.pages.refs > 0).sum())
    cache.pages.compact()
    positions = torch.tensor(length, dtype=torch.int32, device="cuda")
    cache.pages.reserve(list(range(n)), [c + 1 for c in length])
    check = (0, length[0], 1, 0, [1], [length[0]])
    stack.run(cache, cache.batch(list(range(n)), length, [1] * n), state, positions, check=check)
    for status in (cache.sync_status(), cache.pages.sync_status()):
        native.check(status, "longtext")
    full = n * max(-(-c // pages) for c in length)
    print(f"{n} hypotheses of {min(length)}..{max(length)} tokens in {held} pages ({full} unshared), "
          f"{taken / a.steps * 1e3:.2f} ms a step of {n} x {a.nodes} rows, attention off by {stack.error:.1e}")
    cache.close()
    return {"error": stack.error, "held": held, "unshared": full, "length": length}


if __name__ == "__main__":
    main()
