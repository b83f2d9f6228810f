"""attn_fwd_fp8 with scores of any size that FP8 codes give: what counts is how
far a row's scores lie apart, also where its largest has no fraction left."""
import numpy as np
import pytest
import torch

import paper_1812_08011_amd as fp8t
from oracle import lm
from tests.gpu_util import say
from tests.lm_util import check, codes8, offsets, run_attention, value
from tests.test_gpu_attention_special import PLANS

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    fp8t.lib()
    yield


def code(x):
    return {0.0: 0, 1.0: 0x3C, 2.0: 0x40, -1.0: 0xBC, 57344.0: 0x7B, -57344.0: 0xFB}[x]


def compare(q, k, v, cu_q, cu_k, causal, c):
    """The products are multiples of 7 2^13 whose sums fit FP32, so that scores are exact: an
    exponent is off by its distance's rounding, p by 2^-11 (half) twice, the
    sums by n 2^-24; the log-sum-exp by three roundings of itself."""
    ref = lm.attention(value(q), value(k), value(v), cu_q, cu_k, causal, c)
    n = int(np.diff(cu_k).max())
    G = q.shape[1] // k.shape[1]
    top = np.zeros_like(ref["o"])
    for s in range(len(cu_q) - 1):
        at = slice(cu_k[s], cu_k[s + 1])
        for h in range(q.shape[1]):
            top[cu_q[s]:cu_q[s + 1], h] = abs(value(v)[at, h // G]).max(0, initial=0.0)
    err = top * (2.0 ** -10 + (n + 64) * 2.0 ** -24)
    lse = np.where(np.isfinite(ref["lse"]), abs(ref["lse"]), 0) * 3 * 2.0 ** -24 + (n + 64) * 2.0 ** -24
    for kw in PLANS:
        say(f"  plan {kw}")
        got = run_attention(q, k, v, cu_q, cu_k, causal, c, **kw)
        check(f"lse {kw}", got["lse"], ref["lse"], lse)
        check(f"o {kw}", got["o"], ref["o"], err)


@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("c", [1.0, 0.125, 0.1, 0.08838834764, 1e-6, 1e-9, 37.0])
@pytest.mark.parametrize("D", [64, 128])
def test_saturated_queries_and_keys(D, c, sign):
    """Scores of 57344^2 c and their neighbours: equal ones share the row, one
    that is larger by a step takes it, the others' p is 0."""
    say(f"attention, saturated codes, D={D}, scale {c}, sign {sign}")
    c = float(np.float32(c))
    rng = np.random.default_rng(2700 + D)
    lens_q, lens_k = [2, 40, 3], [1500, 40, 700]
    Tq, Tk = sum(lens_q), sum(lens_k)
    q, k = np.zeros((Tq, 4, D), np.uint8), np.zeros((Tk, 2, D), np.uint8)
    v = codes8(rng, (Tk, 2, D))
    q[:, :, 3], k[:, :, 3] = code(57344.0), code(57344.0 * sign)
    q[:, 1:3, 40] = code(1.0)                          # some heads: single keys below the others
    k[rng.random(Tk) < 0.3, :, 40] = code(-57344.0)
    q[:, 2, 41] = code(57344.0)                        # and one key of each sequence above them
    for at in (1499 - 300, 1500 + 1, 1540 + 555):
        k[at, :, 41] = code(57344.0)
    q[0, 3], k[5, 1] = 0, 0                            # a row and a key of zeros
    compare(q, k, v, offsets(lens_q), offsets(lens_k), False, c)


@pytest.mark.parametrize("c", [2.0 ** -4, 2.0 ** -10, 2.0 ** -16])
@pytest.mark.parametrize("step", [0.0, 1.0, 2.0])
@pytest.mark.parametrize("D", [64, 128])
def test_scores_that_grow(D, step, c):
    """The row's largest score moves on, from small to eight saturated products
    (49 2^29), and some keys of each size are another 57344 above."""
    say(f"attention, growing scores, D={D}, step {step}, scale {c}")
    rng = np.random.default_rng(2710 + D)
    T = 900
    q, k, v = np.zeros((4, 2, D), np.uint8), np.zeros((T, 1, D), np.uint8), codes8(rng, (T, 1, D))
    q[:, :, :8] = q[:, :, 20] = code(57344.0)
    for n in range(9):                                 # n of the eight entries are saturated
        k[100 * n:100 * n + 100, 0, :n] = code(57344.0)
    k[::7, 0, 20] = code(step)
    compare(q, k, v, offsets([4]), offsets([T]), True, c)
    compare(q, k[::-1].copy(), v, offsets([4]), offsets([T]), False, c)
