"""Rows that see keys, all of them with a score of -Inf: 0 / 0 in every entry and
a log-sum-exp of -Inf, under every plan and whatever the values are."""
import numpy as np
import pytest
import torch

import paper_1812_08011_amd as fp8t
from tests.gpu_util import say
from tests.lm_util import codes8, offsets, run_attention, value
from tests.test_gpu_attention import INF8
from tests.test_gpu_attention_special import PLANS

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    fp8t.lib()
    yield


@pytest.mark.parametrize("nk", [1, 70, 1500])
@pytest.mark.parametrize("D", [64, 128])
def test_every_score_is_minus_infinity(D, nk):
    say(f"attention, scores of -Inf, D={D}, {nk} keys")
    rng = np.random.default_rng(3000 + nk)
    q, k, v = codes8(rng, (5, 2, D)), codes8(rng, (nk + 9, 1, D)), codes8(rng, (nk + 9, 1, D))
    q[:, :, 2] = 0x3C                                  # 1 times -Inf
    k[:nk, 0, 2] = INF8 | 0x80
    v[nk - 1, 0, 4] = INF8
    cu_q, cu_k = offsets([3, 2]), offsets([nk, 9])
    for kw in PLANS:
        got = run_attention(q, k, v, cu_q, cu_k, False, 0.5, **kw)
        assert np.isneginf(got["lse"][:, :3]).all() and np.isfinite(got["lse"][:, 3:]).all(), kw
        assert np.isnan(value(got["o"][:3])).all() and np.isnan(value(got["o8"][:3])).all(), kw
        assert np.isfinite(value(got["o"][3:])).all(), kw
