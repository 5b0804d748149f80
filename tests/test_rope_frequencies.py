"""Frequencies of the rotary positions against their closed forms."""
import math

import pytest
import torch

from paper_2507_00715_b200.rope import frequencies


def test_plain_and_linear():
    f, a = frequencies(8)
    assert a == 1.0 and f.dtype == torch.float64 and torch.allclose(f, torch.tensor([1.0, 0.1, 0.01, 0.001], dtype=torch.float64))
    g, a = frequencies(8, scaling="linear", factor=4.0)
    assert a == 1.0 and torch.equal(g, f / 4.0)


def test_base_keeps_the_fastest_and_divides_the_slowest():
    f, g = frequencies(64)[0], frequencies(64, scaling="base", factor=8.0)[0]
    assert g[0] == 1.0 and math.isclose(g[-1], f[-1] / 8.0, rel_tol=1e-12) and (g <= f).all()


@pytest.mark.parametrize("kind", ["ramp", "bands"])
def test_parts(kind):
    f, (g, a) = frequencies(128, 500000.0)[0], frequencies(128, 500000.0, kind, 8.0, 8192)
    turns = 8192 * f / (2 * math.pi)
    assert torch.equal(g[turns > 32.5], f[turns > 32.5])
    assert torch.allclose(g[turns < 0.9], f[turns < 0.9] / 8.0, rtol=1e-12)
    ratio = f / g
    assert (ratio[1:] >= ratio[:-1] - 1e-12).all() and a == (0.1 * math.log(8.0) + 1.0 if kind == "ramp" else 1.0)


def test_refusals():
    for kw in (dict(rot_dim=7), dict(rot_dim=0), dict(rot_dim=8, scaling="cubic"), dict(rot_dim=8, scaling="linear", factor=0.5),
               dict(rot_dim=8, scaling="ramp", factor=2.0), dict(rot_dim=8, scaling="bands", factor=2.0, original=100, slow=4.0, fast=2.0)):
        with pytest.raises(ValueError):
            frequencies(**kw)
