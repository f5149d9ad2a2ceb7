"""Scales and codes are those of IEEE quotients, as the definition has it: compared bit for bit with NumPy's fp32 division on
the host (a reciprocal's product, which is what torch makes of a CUDA tensor over a Python number, misses some of them)."""
import numpy as np
import pytest
import torch

import paged_ref as R
from paper_2609_26100_gb300 import native, paged

pytestmark = pytest.mark.gpu
H, D, N = 4, 128, 2048


def definition(x):
    """(codes, s, z) of groups x [..., 64], and whether the product with a reciprocal would give another scale."""
    z = np.clip(x.min(-1), -65504, 65504).astype(np.float16)
    span = x.max(-1) - z.astype(np.float32)
    s, other = (np.clip(q, 0, 65504).astype(np.float16) for q in (span / np.float32(15), span * (np.float32(1) / np.float32(15))))
    sf = np.where(s > 0, s, np.float16(1)).astype(np.float32)[..., None]
    c = np.clip(np.rint((x - z.astype(np.float32)[..., None]) / sf), 0, 15) * (s > 0)[..., None]
    return c.astype(np.int64), s, z, s != other


def groups(kind):
    r = np.random.default_rng(7)
    shape = (N, H, D // 64, 64)
    if kind == "normal":
        return (r.standard_normal(shape) * 10.0 ** r.uniform(-7, 4, shape[:3] + (1,))).astype(np.float32)
    # scales halfway between two fp16 numbers: 0 <= x <= 15 (m + 1/2) 2^e, both ends taken
    m, e = r.integers(1024, 2048, shape[:3] + (1,)), r.integers(-20, -4, shape[:3] + (1,))
    top = (15 * (m + 0.5) * 2.0 ** e).astype(np.float32)
    x = (r.random(shape) * top).astype(np.float32)
    x[..., 5], x[..., 40] = 0, top[..., 0]
    if kind == "halves":  # and values halfway between two codes
        s = ((m + 0.5) * 2.0 ** e).astype(np.float16).astype(np.float32)
        x[..., 6:40] = np.minimum((r.integers(0, 15, shape[:3] + (34,)) + np.float32(0.5)) * s, top)
    return x


@pytest.mark.parametrize("kind", ["normal", "ends", "halves"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_bits(kind, dtype):
    k = torch.from_numpy(groups(kind).reshape(N, H, D)).to(dtype)
    v = k.flip(0)
    pages = N // 64
    c = paged.Kv4Cache.allocate(n_layers=1, n_pages=pages, n_seqs=1, max_pages=pages, n_q_heads=H, n_kv_heads=H, head_dim=D)
    c.pages.reserve([0], [N])
    c.append(0, c.batch([0], [0], [N]), k.cuda(), v.cuda())
    assert c.sync_status() == native.TSS_OK
    blocks = c.pool[0].cpu()[c.table[0].cpu().long()].view(pages, H, -1)
    for side, x in ((0, k), (1, v)):
        codes, s, z, told = definition(x.float().numpy().reshape(N, H, D // 64, 64))
        got = R.params_of(blocks, D, side).permute(0, 2, 1, 3, 4).reshape(N, H, D // 64, 2).numpy()
        assert (got[..., 0] == s).all() and (got[..., 1] == z).all()
        have = R.codes_of(blocks, D, side).permute(0, 2, 1, 3).reshape(N, H, D // 64, 64).numpy()
        assert (have == codes).all()
        if kind != "normal" and dtype == torch.float32:
            assert told.any()
