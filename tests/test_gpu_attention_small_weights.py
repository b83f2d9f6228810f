"""attn_fwd_fp8 where a result comes from keys of small weight alone: the key
that takes the row has values of 0 there."""
import numpy as np
import pytest
import torch

import paper_1812_08011_amd as fp8t
from oracle import lm
from tests.gpu_util import say
from tests.lm_util import check, codes8, offsets, run_attention, value

pytestmark = pytest.mark.gpu
PLANS = [dict(), dict(workspace=False), dict(max_q=300, max_k=8192), dict(max_q=8192)]
ONE = 0x3C


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    fp8t.lib()
    yield


@pytest.mark.parametrize("bits", [10, 20, 26, 30, 33, 36])
@pytest.mark.parametrize("D", [64, 128])
def test_results_of_small_weights(D, bits):
    """One key in three to nine takes the row; the others' p are 2^-bits of it."""
    say(f"attention, weights of 2^-{bits}, D={D}")
    rng = np.random.default_rng(2900 + bits)
    lens_q, lens_k = [1, 40, 2], [3, 9, 5]
    Tq, Tk = sum(lens_q), sum(lens_k)
    q, k, v = np.zeros((Tq, 2, D), np.uint8), np.zeros((Tk, 1, D), np.uint8), codes8(rng, (Tk, 1, D))
    q[:, :, 3] = ONE
    for top in (1, 3 + 7, 12 + 0):
        k[top, 0, 3] = ONE
        v[top] = 0
    c = float(np.float32(bits * np.log(2.0)))
    cu_q, cu_k = offsets(lens_q), offsets(lens_k)
    ref = lm.attention(value(q), value(k), value(v), cu_q, cu_k, False, c)
    for kw in PLANS:
        got = run_attention(q, k, v, cu_q, cu_k, False, c, **kw)
        check(f"o {kw}", got["o"], ref["o"], ref["o_err"])
        check(f"lse {kw}", got["lse"], ref["lse"], ref["lse_err"])


@pytest.mark.parametrize("n", [2, 5, 33, 200])
def test_flat_rows(n):
    """Rows of nearly equal scores: the log-sum-exp's own rounding is all."""
    say(f"attention, flat rows of {n}")
    rng = np.random.default_rng(2950 + n)
    q, k, v = codes8(rng, (60, 4, 16), 0.1), codes8(rng, (n, 2, 16), 0.1), codes8(rng, (n, 2, 16))
    c = float(np.float32(0.01))
    ref = lm.attention(value(q), value(k), value(v), offsets([60]), offsets([n]), False, c)
    for kw in PLANS:
        got = run_attention(q, k, v, offsets([60]), offsets([n]), False, c, **kw)
        check(f"lse {kw}", got["lse"], ref["lse"], ref["lse_err"])
        check(f"o {kw}", got["o"], ref["o"], ref["o_err"])
