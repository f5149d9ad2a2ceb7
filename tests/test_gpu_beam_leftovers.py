"""Beam selection does not depend on what its workspace's memory held before: rows that offer nothing (dead and finished beams) leave
their lists unwritten.  A new workspace gets freed memory full of one word here: a mask's
minus infinities, other floats, ones and zeros."""
import ctypes
import math

import pytest
import torch

from paper_2609_26100_gb300 import beams, native

pytestmark = pytest.mark.gpu


def leave(word, sizes):
    """Freed GPU memory full of this 32-bit word, in blocks of these sizes."""
    cuda = ctypes.CDLL("libcuda.so.1")
    held = []
    for n in sizes:
        for _ in range(32 if n < 1 << 22 else 4):
            at = ctypes.c_uint64()
            assert cuda.cuMemAlloc_v2(ctypes.byref(at), ctypes.c_size_t(n)) == 0
            assert cuda.cuMemsetD32_v2(at, ctypes.c_uint(word), ctypes.c_size_t(n // 4)) == 0
            held.append(at)
    torch.cuda.synchronize()
    for at in held:
        assert cuda.cuMemFree_v2(at) == 0


@pytest.mark.parametrize("word", [0xff800000, 0x7f800000, 0x7fc00000, 0xffffffff, 0], ids=hex)
@pytest.mark.parametrize("rows,vocab,keep", [(8, 32000, 8), (64, 32000, 64), (8, 32000, 128), (256, 131072, 16)])
def test_rows_that_offer_nothing(word, rows, vocab, keep):
    n = 8
    g = torch.Generator(device="cuda").manual_seed(rows + keep)
    x = torch.randn(rows, vocab, generator=g, device="cuda") * 2
    for live in (1, 2):  # the first beam's continuations, then two beams', of each group
        score = torch.full((rows,), -math.inf, device="cuda")
        done = torch.zeros(rows, dtype=torch.int32, device="cuda")
        for b in range(live):
            score[b::n] = -1.0 - b
        score[5::n], done[5::n] = -1e4, 1  # a finished one
        out = torch.empty(rows // n, keep, device="cuda"), *(torch.empty(rows // n, keep, dtype=torch.int32, device="cuda") for _ in range(2))
        lists = max(rows * -(-vocab // 4096), 304)
        leave(word, [lists * keep * 8, lists * 16])
        s = beams.BeamSelector(rows, vocab, keep)
        s.select(x, score, *out, n_beams=n, done=done, end_token=3)
        assert s.sync_status() == native.TSS_OK
        value = (x.double().log_softmax(-1) + score.double()[:, None]).view(rows // n, n, vocab)
        value[:, 5], value[:, 5, 3] = -math.inf, -1e4
        top = value.view(rows // n, -1).topk(keep)
        # (a sum of terms is right to 2^-19: 2^-22 of the fast exponential, 2^-22 of its argument, 24 fp32 additions; candidates
        # closer than that may change places)
        assert ((out[0].double() - top.values).abs() <= top.values.abs() * 2.0 ** -24 + 2.0 ** -19).all()
        place = (out[1].long() - torch.arange(rows // n, device="cuda")[:, None] * n) * vocab + out[2].long()
        assert (place >= 0).all() and all(len(p.unique()) == keep for p in place)
        assert ((value.view(rows // n, -1).gather(1, place) - top.values).abs() <= 2.0 ** -19).all()
