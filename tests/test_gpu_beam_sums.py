"""How right a selection's values are: rows where a few values make up most of the sum, so that its errors are the same ones many times over.

value = score + x - ln S.  Terms that can be chosen are right to 2^-27; the others' sum, relative to itself:
  * their argument x log2(e) - R, rounded twice: 2^-24 |t| twice, times ln 2; with t at most 1/2 in a thread's part of 32 elements and the
    smaller terms' share falling as 2^t, 3.6 2^-24;
  * the fast exponential: 2^-22;
  * a thread's sum, 8 terms each in 4 sums that are then added: 9 roundings of 2^-24;
  * over a chunk's 16 tiles at most: 15 of them;
together under 2^-19 (32 2^-24), which ln S and the value are off by at most.  The value is then rounded once, by 2^-24 of itself, and two
candidates are in the wrong order only where they are closer than 2^-18."""
import pytest
import torch

from paper_2609_26100_gb300 import beams, native

pytestmark = pytest.mark.gpu


def rows_of(kind, rows, vocab, keep, dtype, g):
    floor = -1 - 6 * torch.rand(rows, 1, generator=g, device="cuda")
    some = torch.randint(0, 8, (rows, vocab), generator=g, device="cuda")
    at = torch.arange(vocab, device="cuda")
    x = {"one value": lambda: floor.repeat(1, vocab), "two": lambda: floor - 2.0 * (some & 1), "eight": lambda: floor - 0.5 * some,
         # (one larger element in every 16 neighbours and in every thread's part of a tile)
         "one larger": lambda: torch.where((at % 16 == 0)[None], floor + 2.43, floor)}[kind]()
    peaks = torch.randint(vocab, (max(2, keep // 2),), generator=g, device="cuda")
    x[:, peaks] = 3.0
    return x.to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("kind", ["one value", "two", "eight", "one larger"])
@pytest.mark.parametrize("rows,n_beams,vocab,keep", [(8, 2, 2000, 4), (64, 8, 32000, 8), (512, 8, 50021, 16), (256, 32, 131072, 32)])
def test_bound(dtype, kind, rows, n_beams, vocab, keep):
    g = torch.Generator(device="cuda").manual_seed(vocab + keep)
    x = rows_of(kind, rows, vocab, keep, dtype, g)
    score = torch.randn(rows, generator=g, device="cuda") * 1e-6  # (beams whose order hangs on the sums)
    n = rows // n_beams
    out = torch.empty(n, keep, device="cuda"), *(torch.empty(n, keep, dtype=torch.int32, device="cuda") for _ in range(2))
    s = beams.BeamSelector(rows, vocab, keep)
    s.select(x, score, *out, n_beams=n_beams)
    assert s.sync_status() == native.TSS_OK
    bound = 2.0 ** -19
    for i in range(n):
        part = slice(i * n_beams, (i + 1) * n_beams)
        v = (x[part].double().log_softmax(-1) + score[part].double()[:, None]).view(-1)
        top = v.topk(keep).values
        place = (out[1][i].long() - i * n_beams) * vocab + out[2][i].long()
        assert (place >= 0).all() and place.unique().numel() == keep
        mine = v[place]
        assert ((out[0][i].double() - mine).abs() <= mine.abs() * 2.0 ** -24 + bound).all()
        assert (mine[:-1] - mine[1:] >= -2 * bound).all() and (mine >= top - 2 * bound).all()
        # equal logits of one row, whose values are equal: the lower token first
        same = (place[:-1] // vocab == place[1:] // vocab) & (mine[:-1] == mine[1:])
        assert (place[:-1] < place[1:])[same].all()
