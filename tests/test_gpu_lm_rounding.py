"""Results in FP16 are one rounding of the FP32 value at every magnitude:
rotary_embed on values that it only converts, against the quantizer's
definition, in places that whole loads take and in rows' ends."""
import numpy as np
import pytest
import torch

import oracle
import paper_1812_08011_amd as fp8t
from tests.gpu_util import DEV, dev, host, say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    fp8t.lib()
    yield


def near_ties():
    """Floats at, just beside and far from the ties between FP16 values, from
    below the smallest to above the largest."""
    rng = np.random.default_rng(60)
    n = np.arange(0, 1030)
    ties = [(n + 0.5) * 2.0 ** -39, n * 2.0 ** -39]
    for e in (-30, -29, -24, -1, 0, 5, 29, 30, 31):
        ties.append((512 + rng.integers(0, 512, 200) + 0.5) * 2.0 ** (e - 9))
    x = np.concatenate(ties)
    d = np.concatenate([[0.0], 2.0 ** -np.arange(1.0, 24), -2.0 ** -np.arange(1.0, 24)])
    x = (x[:, None] * (1 + d)).ravel().astype(np.float32)
    x = np.concatenate([x, np.nextafter(x, np.float32(np.inf)), np.nextafter(x, np.float32(0)),
                        2.0 ** rng.uniform(-149, 33, 5000).astype(np.float32),
                        np.array([0.0, 2.0 ** -149, 2.0 ** -126, np.inf, np.nan], np.float32)])
    x = np.concatenate([x, -x])
    rng.shuffle(x)
    return x


@pytest.mark.parametrize("D", [8, 16, 24, 37, 100])
def test_every_magnitude_is_rounded_once(D):
    say(f"rounding to FP16, D={D}")
    x = near_ties()
    x = x[:x.size // D * D].reshape(-1, 1, D)
    T = len(x)
    y = torch.empty((T, 1, D), dtype=torch.uint16, device=DEV)
    fp8t.rotary_embed(dev(x), dev(np.zeros(T, np.int64)), dev(np.zeros(0)), y)
    got, want = host(y), oracle.fp16_quantize(x)
    bad = np.argwhere(got != want)
    assert len(bad) == 0, [(x[tuple(i)], got[tuple(i)], want[tuple(i)]) for i in bad[:5]]
