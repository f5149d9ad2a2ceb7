"""Example: several continuations of one long prompt over a paged 4-bit KV cache.

    python -m paper_2609_26100_gb300.longtext [--prompt 3000] [--steps 6] [--hypotheses 4] [--layers 4]

A stack of attention layers with random weights (head norms, rotary positions stretched for a long
context, grouped heads; every second layer sees a window and the first tokens) decodes speculatively:

  * the prompt enters in chunks of 128 rows: project, norm and rotate (tss_qk_rope), append
    (tss_paged_append), attend (tss_paged_attention);
  * its pages are shared by all hypotheses (tss_pages_fork), a part-filled last page is copied;
  * a step scores a draft tree for every hypothesis, takes a path of it, and appends the path's rows in
    order over the block's; pages past it are given back (tss_pages_free);
  * every second step the worse half is dropped and forked from the better half; at the end the pool is
    made dense (tss_pages_compact).

It checks the attention against a plain computation on the values read back (tss_paged_read) and prints the
error and the time of a step.
"""
from __future__ import annotations

import argparse
import random
import time

import torch

from . import native, paged

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

    def run(self, cache: paged.Kv4Cache, batch, x, positions, mask=None, check=None):
        """Rows x of the batch's blocks through all layers, their keys and values appended on the way; the
        outputs and each layer's rotated keys and values.  check: a request whose first layer is compared with
        a plain computation."""
        kept = []
        for layer in range(self.layers):
            n = x.shape[0]
            rows = torch.nn.functional.linear(x / x.float().square().mean(-1, keepdim=True).sqrt().bfloat16(), self.wqkv[layer])
            rows = rows.view(n, self.hq + 2 * self.hk, self.d)
            q, k, v = rows[:, :self.hq], rows[:, self.hq:self.hq + self.hk], rows[:, self.hq + self.hk:]
            native.qk_rope(native.rope_args(q, k, q, k, positions, self.table, q_gain=self.gains[layer][0],
                                            k_gain=self.gains[layer][1]))
            cache.append(layer, batch, k, v)
            out = torch.empty(n, self.hq, self.d, dtype=x.dtype, device=x.device)
            near = {"window": WINDOW, "sinks": SINKS} if layer % 2 else {}
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


def main(argv=None) -> dict:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--prompt", type=int, default=3000)
    ap.add_argument("--steps", type=int, default=6)
    ap.add_argument("--hypotheses", type=int, default=4)
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--nodes", type=int, default=12, help="rows of a draft tree, its root included")
    ap.add_argument("--seed", type=int, default=1)
    a = ap.parse_args(argv)
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
