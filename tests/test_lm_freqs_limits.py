"""rotary_freqs refuses what would give angles that are not numbers."""
import math

import numpy as np
import pytest

from paper_1812_08011_amd.lm import rotary_freqs


@pytest.mark.parametrize("bad", [dict(factor=math.nan), dict(factor=math.inf),
                                 dict(slow_turns=32.0, fast_turns=32.0), dict(slow_turns=40.0),
                                 dict(fast_turns=math.nan)], ids=str)
def test_refusals(bad):
    with pytest.raises(ValueError):
        rotary_freqs(64, **{**dict(scaling="by_parts", factor=4.0), **bad})


def test_what_is_taken_is_finite():
    for scaling in (None, "linear", "base", "by_parts"):
        for factor in (1.0, 3.5, 1e6):
            f, m = rotary_freqs(64, scaling=scaling, factor=factor)
            assert np.isfinite(f).all() and (f > 0).all() and math.isfinite(m)
