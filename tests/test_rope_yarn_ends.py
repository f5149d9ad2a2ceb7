"""tss_rope_frequencies, YARN: where the slowest pairs turn more than once within the original context, no pair is divided
by the whole factor, and the ramp ends where its index says, past the last pair."""
import math

import pytest

from paper_2609_26100_gb300 import build, native


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build()


@pytest.mark.parametrize("rot", [64, 128])
@pytest.mark.parametrize("theta,original", [(1e4, 2048.0), (1e4, 4096.0), (1e4, 65536.0), (1e4, 131072.0), (1e4, 1e6), (1e4, 1e12 - 1), (5e5, 8192.0),
                                            (1.5, 4096.0)])
@pytest.mark.parametrize("factor", [1.0, 8.0, 40.0])
def test_definition(rot, theta, original, factor):
    f, a = native.rope_frequencies(rot, theta, "yarn", factor, original)
    assert abs(a - (0.1 * math.log(factor) + 1)) < 1e-15
    index = [rot * math.log(original / (2 * math.pi * t)) / (2 * math.log(theta)) for t in (32, 1)]
    lo, hi = max(0, math.floor(index[0])), min(rot - 1, math.ceil(index[1]))
    step = 1 / (hi - lo) if hi > lo else 0.0  # (a ramp that begins past its end divides nothing)
    for i, x in enumerate(f):
        y = theta ** (-2 * i / rot)
        r = 0.0 if i <= lo else 1.0 if i >= hi else (i - lo) / (hi - lo)
        assert abs(x - (y * (1 - r) + y / factor * r)) <= 1e-13 * y, i
        turns = original * y / (2 * math.pi)
        if turns > 32:
            assert x >= y * (1 - (1 - 1 / factor) * step - 1e-13), i  # (the ramp begins at a whole index: less than a step of it)
        if turns > 1 and factor > 1:
            assert x > y / factor * (1 + 1e-9), i
        if turns < 1 and i >= hi:
            assert abs(x - y / factor) <= 1e-13 * y, i


def test_the_slowest_pair_of_a_long_original_context():
    """theta 1e4, 131072 tokens: pair 63 of 64 turns 2.4 times and stands 18 of 25 steps up the ramp."""
    f, _ = native.rope_frequencies(128, 1e4, "yarn", 8.0, 131072.0)
    y = 1e4 ** (-126 / 128)
    assert abs(f[63] / y - (1 - 18 / 25 * 7 / 8)) < 1e-12
