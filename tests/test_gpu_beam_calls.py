"""Ways of calling the operators for several continuations: a whole step captured and replayed on inputs that change, two captured steps that
share workspaces, steps on two streams at once, tensors of another GPU and calls while another one is current (a second GPU is pretended:
get_device() and current_device() answer 1).  Results are compared bit for bit with those of eager calls one after another."""
import pytest
import torch

from paper_2609_26100_gb300 import beams, native, paged

pytestmark = pytest.mark.gpu
ROWS, HQ, HK, D, VOCAB, SHARED = 12, 8, 2, 128, 777, 200


class Step:
    """A step of a search of two texts: its cache, books and selector, inputs and outputs."""

    def __init__(self, seed, dtype=torch.bfloat16):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.g, self.dtype, self.length = g, dtype, [SHARED] * 6 + [SHARED + 55] * 6
        self.cache = paged.Kv4Cache.allocate(n_layers=1, n_pages=80, n_seqs=ROWS, max_pages=8, n_q_heads=HQ, n_kv_heads=HK, head_dim=D, shared_rows=ROWS)
        self.selector = beams.BeamSelector(ROWS, VOCAB, 6)
        self.table = torch.rand(400, D // 2, 2, generator=g, device="cuda")
        self.gain = (1 + 0.1 * torch.randn(D, generator=g, device="cuda")).to(dtype)
        self.q, self.k, self.v, self.logits = self.normal(ROWS, HQ, D), self.normal(ROWS, HK, D), self.normal(ROWS, HK, D), self.normal(ROWS, VOCAB)
        self.q_out, self.out = torch.empty_like(self.q), torch.empty_like(self.q)
        self.score, self.score_out = torch.zeros(ROWS, device="cuda"), torch.empty(2, 6, device="cuda")
        self.parent, self.token = (torch.empty(2, 6, dtype=torch.int32, device="cuda") for _ in range(2))
        self.positions = torch.tensor(self.length, dtype=torch.int32, device="cuda")
        for t in (0, 6):
            n = self.length[t]
            self.cache.pages.reserve([t], [n])
            self.cache.append(0, self.cache.batch([t], [0], [n]), self.normal(n, HK, D), self.normal(n, HK, D))
            self.cache.pages.fork([t] * 5, list(range(t + 1, t + 6)), [n] * 5)
        c = self.cache
        self.state = [x for x in (c.pool, c.table, c.pages.held, c.pages.refs)]
        torch.cuda.synchronize()
        self.saved = [x.clone() for x in self.state]

    def normal(self, *shape):
        return torch.randn(*shape, generator=self.g, device="cuda").to(self.dtype)

    def inputs(self, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        for x in (self.q, self.k, self.v, self.logits, self.score):
            x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
        for x, y in zip(self.state, self.saved):
            x.copy_(y)

    def run(self):
        c, seqs, tokens = self.cache, list(range(ROWS)), [n + 1 for n in self.length]
        c.pages.reserve(seqs, tokens)
        batch = c.batch(seqs, self.length, [1] * ROWS)
        c.append_rope(0, batch, native.rope_args(self.q, self.k, self.q_out, None, self.positions, self.table, q_gain=self.gain, k_gain=self.gain,
                                                 to_pages=True), self.v)
        c.attention_shared(0, batch, c.groups([6, 6], [self.length[0], self.length[6]]), self.q_out, self.out)
        self.selector.select(self.logits, self.score, self.score_out, self.parent, self.token, n_beams=6)
        c.pages.reorder(seqs, self.parent.view(-1), tokens)

    def results(self):
        torch.cuda.synchronize()
        assert [x.sync_status() for x in (self.cache, self.cache.pages, self.selector)] == [native.TSS_OK] * 3
        return [x.clone() for x in (*self.state, self.q_out, self.out, self.score_out, self.parent, self.token)]

    def eager(self, seed):
        self.inputs(seed)
        self.run()
        return self.results()


def same(a, b):
    return all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a, b))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_captured_steps_that_share_workspaces(dtype):
    s = Step(1, dtype)
    want = {seed: s.eager(seed) for seed in (10, 11, 12)}
    assert not same(want[10], want[11])
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            s.run()
        graphs.append(graph)
    for i, seed in enumerate((11, 10, 12, 12, 10)):
        s.inputs(seed)
        graphs[i % 2].replay()
        assert same(s.results(), want[seed]), (i, seed)
    assert same(s.eager(11), want[11])  # (and eager calls beside living graphs)


def test_two_streams_at_once():
    steps = [Step(seed) for seed in (2, 3)]
    want = [s.eager(20) for s in steps]
    streams = [torch.cuda.Stream() for _ in steps]
    for _ in range(5):
        for s in steps:
            s.inputs(20)
        torch.cuda.synchronize()
        for s, stream in zip(steps, streams):
            with torch.cuda.stream(stream):
                for _ in range(3):  # (each from the state that the last one left)
                    for x, y in zip(s.state, s.saved):
                        x.copy_(y)
                    s.run()
        assert all(same(s.results(), w) for s, w in zip(steps, want))


class Elsewhere(torch.Tensor):
    def get_device(self):
        return 1


def elsewhere(t):
    return t.as_subclass(Elsewhere)


def test_another_device(monkeypatch):
    s = Step(4)
    c, batch = s.cache, s.cache.batch(list(range(ROWS)), s.length, [1] * ROWS)
    groups = c.groups([6, 6], [SHARED, SHARED])
    args = native.rope_args(s.q, s.k, s.q_out, None, s.positions, s.table, to_pages=True)
    outs = (s.score_out, s.parent, s.token)
    calls = [lambda: c.append_rope(0, batch, args, s.v), lambda: c.attention_shared(0, batch, groups, s.q_out, s.out),
             lambda: s.selector.select(s.logits, s.score, *outs, n_beams=6), lambda: s.selector.sync_status(),
             lambda: c.pages.reorder(list(range(ROWS)), torch.arange(ROWS, dtype=torch.int32, device="cuda"), s.length)]
    torch.cuda.synchronize()
    with monkeypatch.context() as m:
        m.setattr(torch.cuda, "current_device", lambda: 1)
        for call in calls:
            with pytest.raises(ValueError):
                call()
    for bad in (lambda: c.append_rope(0, batch, args, elsewhere(s.v)),
                lambda: native.rope_args(s.q, elsewhere(s.k), s.q_out, None, s.positions, s.table, to_pages=True),
                lambda: c.attention_shared(0, batch, groups, elsewhere(s.q_out), s.out),
                lambda: s.selector.select(elsewhere(s.logits), s.score, *outs, n_beams=6),
                lambda: s.selector.select(s.logits, elsewhere(s.score), *outs, n_beams=6),
                lambda: s.selector.select(s.logits, s.score, s.score_out, elsewhere(s.parent), s.token, n_beams=6),
                lambda: c.pages.reorder(list(range(ROWS)), elsewhere(torch.zeros(ROWS, dtype=torch.int32, device="cuda")), s.length)):
        with pytest.raises(ValueError):
            bad()
    assert all(torch.equal(x, y) for x, y in zip(s.state, s.saved))
    s.results()
