"""Kv4Cache.batch on the host: what it holds, and that numbers past 32 bits are refused rather than wrapped."""
import ctypes

import pytest
import torch

from paper_2609_26100_gb300 import paged


def held(address, n):
    return list((ctypes.c_int32 * n).from_address(address))


def test_what_a_batch_holds():
    b = paged.Kv4Cache.batch([3, 0], (2 ** 31 - 1, 7), torch.tensor([5, 0]))
    assert (b.n_req, b.rows) == (2, 5)
    assert [held(x, 2) for x in (b.seq, b.first, b.n_tokens)] == [[3, 0], [2 ** 31 - 1, 7], [5, 0]]


@pytest.mark.parametrize("big", [2 ** 31, 2 ** 32, 2 ** 32 + 1, -2 ** 31 - 1, 2 ** 64])
@pytest.mark.parametrize("which", range(3))
def test_numbers_past_32_bits(big, which):
    args = [[0, 1], [5, 6], [7, 8]]
    args[which][1] = big
    with pytest.raises(OverflowError):
        paged.Kv4Cache.batch(*args)
