"""README.md's search over the paged cache runs as it is written: every step's tokens have pages, also past a page's end, and nothing is
recorded.  The stack is cut to two layers; projections and logits are random tensors of the shapes that the text names."""
import os
import re
import types

import pytest
import torch

from paper_2609_26100_gb300 import native, paged

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_search_of_the_readme():
    with open(os.path.join(ROOT, "README.md")) as f:
        block, = [x for x in re.findall(r"```python\n(.*?)```", f.read(), re.S) if "append_rope" in x]
    made = []

    class Cache(paged.Kv4Cache):
        @classmethod
        def allocate(cls, **kw):
            made.append(paged.Kv4Cache.allocate(**{**kw, "n_layers": 2, "n_pages": 64}))
            return made[-1]

    g = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    freq, factor = native.rope_frequencies(128, 10000.0)
    table = torch.empty(512, 64, 2, device="cuda")
    native.rope_table(freq, table, factor)
    beams = 8
    score = torch.full((beams,), -torch.inf, device="cuda")
    score[0] = 0.0
    prompt, steps = 120, 80
    names = dict(native=native, paged=types.SimpleNamespace(Kv4Cache=Cache), torch=torch, layers=range(2), layer=0, prompt=prompt, steps=steps, length=prompt, table=table,
                 q_gain=None, k_gain=None, q=rnd(beams, 32, 128).bfloat16(), k=rnd(beams, 8, 128).bfloat16(), v=rnd(beams, 8, 128).bfloat16(),
                 out=torch.empty(beams, 32, 128, dtype=torch.bfloat16, device="cuda"), logits=rnd(beams, 32000), score=score, score_out=torch.empty(1, beams, device="cuda"),
                 parent=torch.empty(1, beams, dtype=torch.int32, device="cuda"), token=torch.empty(1, beams, dtype=torch.int32, device="cuda"),
                 done=torch.zeros(beams, dtype=torch.int32, device="cuda"), positions=torch.full((beams,), prompt, dtype=torch.int32, device="cuda"))
    exec(compile(block, "README.md", "exec"), names)
    cache, = made
    assert (cache.sync_status(), cache.pages.sync_status(), names["best"].sync_status()) == (native.TSS_OK,) * 3
    held = (prompt + steps + 63) // 64
    assert cache.pages.held.tolist() == [held] * beams and (cache.table[:, :held] >= 0).all()
    assert (cache.table[:, 0] == cache.table[0, 0]).all()                 # the prompt's whole page is one
    assert len(cache.table[:, held - 1].unique()) == beams                # the last, part-filled one is every beam's own
