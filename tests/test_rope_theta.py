"""Bases that give no frequencies are refused by name."""
import pytest
import torch

from paper_2507_00715_b200.rope import frequencies


@pytest.mark.parametrize("theta", [0.0, -10000.0, float("nan"), float("inf")])
@pytest.mark.parametrize("kw", [{}, dict(scaling="linear", factor=2.0), dict(scaling="base", factor=2.0),
                                dict(scaling="ramp", factor=2.0, original=4096), dict(scaling="bands", factor=2.0, original=4096)])
def test_refused(theta, kw):
    with pytest.raises(ValueError, match="theta"):
        frequencies(64, theta, **kw)


@pytest.mark.parametrize("theta", [1.0, 0.5])
def test_a_ramp_needs_pairs_that_slow_down(theta):
    with pytest.raises(ValueError, match="theta"):
        frequencies(64, theta, "ramp", 2.0, 4096)
    assert torch.isfinite(frequencies(64, theta)[0]).all()


@pytest.mark.parametrize("factor", [float("nan"), float("inf")])
def test_factor(factor):
    for kind in ("linear", "base", "ramp", "bands"):
        with pytest.raises(ValueError, match="factor"):
            frequencies(64, 10000.0, kind, factor, 4096)
