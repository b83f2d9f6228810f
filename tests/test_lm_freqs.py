"""Angles per position for rotary_embed (paper_1812_08011_amd.lm.rotary_freqs)."""
import math

import numpy as np
import pytest

from paper_1812_08011_amd.lm import rotary_freqs


def test_plain_and_linear():
    f, m = rotary_freqs(8, 10000.0)
    assert m == 1.0 and f.dtype == np.float64
    assert np.allclose(f, [1.0, 0.1, 0.01, 0.001])
    g, m = rotary_freqs(8, 10000.0, "linear", 4.0)
    assert m == 1.0 and np.allclose(g, f / 4.0)


def test_base_scaling_keeps_the_fastest_and_slows_the_slowest():
    f, _ = rotary_freqs(64)
    g, _ = rotary_freqs(64, scaling="base", factor=8.0)
    assert g[0] == 1.0 and np.isclose(g[-1], f[-1] / 8.0)
    assert (np.diff(g / f) < 0).all()


def test_by_parts():
    f, _ = rotary_freqs(128)
    g, m = rotary_freqs(128, scaling="by_parts", factor=16.0, original_length=4096)
    assert np.isclose(m, 0.1 * math.log(16.0) + 1.0)
    turns = f * 4096 / (2 * math.pi)
    assert np.array_equal(g[turns >= 32], f[turns >= 32])
    assert np.allclose(g[turns <= 1], f[turns <= 1] / 16.0)
    between = (turns > 1) & (turns < 32)
    assert between.any() and ((g < f) & (g > f / 16.0))[between].all()
    assert np.array_equal(rotary_freqs(128, scaling="by_parts", factor=1.0)[0], f)


@pytest.mark.parametrize("bad", [dict(R=7), dict(R=0), dict(R=8, scaling="other"),
                                 dict(R=8, scaling="linear", factor=0.5)])
def test_refusals(bad):
    with pytest.raises(ValueError):
        rotary_freqs(**bad)
