"""Rotary arguments whose tensors are missing are refused with ValueError."""
import pytest
import torch

from paper_2609_26100_gb300 import native

pytestmark = pytest.mark.gpu


def test_rotary_tensors_that_are_missing():
    x = torch.ones(2, 1, 64, device="cuda")
    table, pos = torch.zeros(4, 32, 2, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    for args in ((x, None, None, None, pos, table), (None, x, None, None, pos, table), (x, None, x, None, None, table), (None, None, None, None, pos, table)):
        with pytest.raises(ValueError):
            native.rope_args(*args)
