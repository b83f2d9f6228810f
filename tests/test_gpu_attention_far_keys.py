"""attn_fwd_fp8 where a row's first keys lie far below the others: the scores of
those that count keep their fractions, whatever came before them."""
import numpy as np
import pytest
import torch

import paper_1812_08011_amd as fp8t
from tests.gpu_util import say
from tests.lm_util import codes8, offsets, run_attention, value
from tests.test_gpu_attention_large_scores import code, compare
from tests.test_gpu_attention_special import PLANS

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    fp8t.lib()
    yield


@pytest.mark.parametrize("first", [31, 64, 200, 777])
@pytest.mark.parametrize("c", [0.5, 0.0883883])
@pytest.mark.parametrize("D", [64, 128])
def test_far_keys_come_first(D, c, first):
    """The first keys at -57344^2 c, the others at small whole numbers times c:
    exact products and sums all."""
    say(f"attention, {first} far keys first, D={D}, scale {c}")
    rng = np.random.default_rng(2800 + D)
    c, lens_q, lens_k = float(np.float32(c)), [3, 40], [1500, 900]
    Tq, Tk = sum(lens_q), sum(lens_k)
    q, k, v = np.zeros((Tq, 2, D), np.uint8), np.zeros((Tk, 1, D), np.uint8), codes8(rng, (Tk, 1, D))
    small = np.array([code(x) for x in (0.0, 1.0, 2.0, -1.0)], np.uint8)
    q[:, :, 8:24] = code(1.0)
    k[:, 0, 8:24] = small[rng.integers(0, 4, (Tk, 16))]
    q[:, :, 3] = code(57344.0)
    for start in (0, 1500):
        k[start:start + first, 0, 3] = code(-57344.0)
        k[start:start + first, 0, 8:24] = 0
    compare(q, k, v, offsets(lens_q), offsets(lens_k), True, c)


@pytest.mark.parametrize("c", [1e-3, 1e20, 1e30, 3.4e38])
def test_the_largest_scales(c):
    """Scales up to FP32's largest: one key takes each row, wherever it lies."""
    say(f"attention, scale {c}")
    rng = np.random.default_rng(2810)
    q, k = np.zeros((1, 1, 64), np.uint8), np.zeros((900, 1, 64), np.uint8)
    v = codes8(rng, (900, 1, 64))
    q[0, 0, :2] = code(57344.0)
    k[:, 0, 0] = code(-57344.0)
    k[700, 0, 0] = code(-1.0)
    for kw in PLANS:
        got = run_attention(q, k, v, offsets([1]), offsets([900]), True, c, **kw)
        assert np.array_equal(value(got["o8"][0]), value(v[700])), kw
