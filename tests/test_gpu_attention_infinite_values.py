"""Infinite values under every plan of attn_fwd_fp8: a row that sees one has
that infinity, whatever its weight and whichever workgroup met it."""
import numpy as np
import pytest
import torch

import paper_1812_08011_amd as fp8t
from tests.gpu_util import say
from tests.lm_util import codes8, offsets, value
from tests.test_gpu_attention import INF8
from tests.test_gpu_attention_special import compare

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    fp8t.lib()
    yield


@pytest.mark.parametrize("gap", [0.0, 30.0, 400.0])
@pytest.mark.parametrize("D", [64, 128])
def test_infinite_values_of_any_weight(D, gap):
    """A row that sees an infinite value has that infinity, however small the
    value's weight is; two of opposite signs give NaN.  gap: how far the scores
    of the infinite values' keys lie below the others'."""
    say(f"attention, infinite values {gap} below, D={D}")
    rng = np.random.default_rng(2300 + D)
    lens_q, lens_k = [3, 150], [1500, 700]
    q = np.zeros((153, 2, D), np.uint8)
    q[:, :, 0] = codes8(rng, (153, 2)) & 0x03 | 0x3C        # the first entry from 1 to 1.75
    k = codes8(rng, (2200, 1, D), 0.25)
    v = codes8(rng, (2200, 1, D))
    low = np.array([5, 700, 1499, 1500 + 3, 1500 + 333, 1500 + 560])
    p8 = value(np.arange(0x7C, dtype=np.uint8))
    k[low, 0, 0] = 0x80 | int(np.argmin(abs(p8 - gap)))
    v[low, 0, 7] = INF8
    v[700, 0, 9] = INF8 | 0x80
    v[1499, 0, 9] = INF8
    v[1500 + 333, 0, D - 1] = INF8 | 0x80
    compare(q, k, v, offsets(lens_q), offsets(lens_k), True, 1.0)
