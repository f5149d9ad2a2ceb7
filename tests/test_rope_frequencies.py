"""tss_rope_frequencies on the host: the scalings' formulas and its refusals."""
import math

import pytest

from paper_2609_26100_gb300 import build, native


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build()


def plain(rot, theta):
    return [theta ** (-2 * i / rot) for i in range(rot // 2)]


def close(a, b):
    return len(a) == len(b) and all(abs(x - y) <= 1e-13 * abs(y) for x, y in zip(a, b))


@pytest.mark.parametrize("rot,theta", [(2, 10000.0), (64, 10000.0), (128, 500000.0)])
def test_unscaled_linear_and_ntk(rot, theta):
    f, a = native.rope_frequencies(rot, theta)
    assert close(f, plain(rot, theta)) and a == 1.0
    f, a = native.rope_frequencies(rot, theta, "linear", 4.0)
    assert close(f, [x / 4.0 for x in plain(rot, theta)]) and a == 1.0
    if rot >= 4:
        f, a = native.rope_frequencies(rot, theta, "ntk", 4.0)
        assert close(f, plain(rot, theta * 4.0 ** (rot / (rot - 2)))) and a == 1.0
        assert abs(f[-1] * 4.0 / plain(rot, theta)[-1] - 1) < 1e-12  # the slowest pair is stretched by the factor


def test_yarn():
    rot, theta, factor, original = 128, 10000.0, 16.0, 4096.0
    f, a = native.rope_frequencies(rot, theta, "yarn", factor, original)
    assert abs(a - (0.1 * math.log(factor) + 1)) < 1e-15
    lo = math.floor(rot * math.log(original / (2 * math.pi * 32)) / (2 * math.log(theta)))
    hi = math.ceil(rot * math.log(original / (2 * math.pi)) / (2 * math.log(theta)))
    for i, (x, y) in enumerate(zip(f, plain(rot, theta))):
        r = min(1.0, max(0.0, (i - lo) / (hi - lo)))
        assert abs(x - (y * (1 - r) + y / factor * r)) <= 1e-13 * y
    assert f[0] == 1.0 and abs(f[-1] * factor / plain(rot, theta)[-1] - 1) < 1e-12


def test_bands():
    rot, theta, factor, original = 128, 500000.0, 8.0, 8192.0
    f, a = native.rope_frequencies(rot, theta, "bands", factor, original)
    assert a == 1.0
    kinds = set()
    for x, y in zip(f, plain(rot, theta)):
        wave = 2 * math.pi / y
        if wave < original / 4:
            want, kind = y, "kept"
        elif wave > original:
            want, kind = y / factor, "divided"
        else:
            keep = (original / wave - 1) / (4 - 1)
            want, kind = keep * y + (1 - keep) * y / factor, "between"
        kinds.add(kind)
        assert abs(x - want) <= 1e-13 * want
    assert len(kinds) == 3


@pytest.mark.parametrize("args", [(0, 1e4), (63, 1e4), (64, 1.0), (64, math.nan), (64, 1e4, "linear", 0.5), (64, 1e4, "ntk", math.inf),
                                  (2, 1e4, "ntk", 2.0), (64, 1e4, "yarn", 2.0, 0.0), (64, 1e4, "bands", 2.0, math.nan)])
def test_refusals(args):
    with pytest.raises(native.TssError) as e:
        native.rope_frequencies(*args)
    assert e.value.status == native.TSS_ERR_INVALID_ARG
