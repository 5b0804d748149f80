"""The ramp between kept and divided rotary frequencies against its closed form, pair by pair."""
import math

import pytest

from paper_2507_00715_b200.rope import frequencies


def expected(rot, theta, factor, original, slow, fast):
    """Loops and scalars: a pair's number at `n` turns is where original * theta^(-2 x / rot) = 2 pi n."""
    first, last = (math.floor if n == fast else math.ceil for n in (fast, slow))
    first, last = (end(rot / 2 * math.log(original / (2 * math.pi * n), theta)) for end, n in ((first, fast), (last, slow)))
    out = []
    for i in range(rot // 2):
        w = 1.0 if i <= first else 0.0 if i >= last else (last - i) / (last - first)
        f = theta ** (-2.0 * i / rot)
        out.append(w * f + (1.0 - w) * f / factor)
    return out


@pytest.mark.parametrize("rot,theta,factor,original,slow,fast", [
    (128, 10000.0, 8.0, 131072, 1.0, 32.0),    # the slowest pair makes 2.4 turns: it is not divided by the whole factor
    (128, 10000.0, 4.0, 131072, 1.0, 32.0), (128, 1e6, 4.0, 32768, 1.0, 32.0), (128, 500000.0, 8.0, 8192, 1.0, 32.0),
    (64, 10000.0, 16.0, 4096, 1.0, 32.0), (20, 10000.0, 2.0, 2048, 2.0, 16.0), (2, 10000.0, 4.0, 4096, 1.0, 32.0),
    (128, 10000.0, 4.0, 128, 1.0, 32.0),       # the fastest pair makes 20 turns: between kept and divided
    (128, 10000.0, 4.0, 128, 32.0, 64.0),      # less than `slow` turns everywhere: every pair is divided
    (128, 10000.0, 4.0, 10 ** 9, 1.0, 32.0)])  # more than `fast` turns everywhere: every pair is kept
def test_every_pair(rot, theta, factor, original, slow, fast):
    got, amplitude = frequencies(rot, theta, "ramp", factor, original, slow, fast)
    want = expected(rot, theta, factor, original, slow, fast)
    assert len(got) == rot // 2 and amplitude == 0.1 * math.log(factor) + 1.0
    for i, (x, y) in enumerate(zip(got.tolist(), want)):
        assert math.isclose(x, y, rel_tol=1e-12), (i, x, y)
        turns = original * theta ** (-2.0 * i / rot) / (2.0 * math.pi)
        whole = theta ** (-2.0 * i / rot)
        if turns > fast:
            assert x == pytest.approx(whole, rel=1e-14)
        if turns < slow:
            assert x == pytest.approx(whole / factor, rel=1e-14)


def test_known_weights():
    """rot_dim 128, theta 10000, original 131072: the ends are pairs 45.03 and 69.11, so 45 and 70; pair 63 keeps 7 / 25."""
    got = frequencies(128, 10000.0, "ramp", 4.0, 131072)[0]
    assert math.isclose(float(got[63]) / 10000.0 ** (-126 / 128), 7 / 25 + 18 / 25 / 4.0, rel_tol=1e-12)
