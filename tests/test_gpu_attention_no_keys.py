"""Attention calls without a single key, or without a query: every row has o =
+0 and lse = -Inf, every gradient is +0, under every plan."""
import numpy as np
import pytest
import torch

import paper_1812_08011_amd as fp8t
from tests.gpu_util import say
from tests.lm_util import codes8, run_attention

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    fp8t.lib()
    yield


@pytest.mark.parametrize("kw", [dict(), dict(max_q=8192), dict(max_q=8192, max_k=8192),
                                dict(max_q=8192, workspace=False)], ids=str)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens_q", [[5], [200], [70, 3]], ids=str)
def test_no_keys(lens_q, D, causal, kw):
    say(f"attention without keys {lens_q} D={D} causal={causal} {kw}")
    rng = np.random.default_rng(2400)
    T, none = sum(lens_q), np.zeros((0, 2, D), np.uint8)
    cu_q = np.concatenate([[0], np.cumsum(lens_q)])
    q, e = codes8(rng, (T, 4, D)), codes8(rng, (T, 4, D))
    got = run_attention(q, none, none, cu_q, np.zeros(len(cu_q), np.int64), causal, 0.125, e, **kw)
    for n in ("o", "o8", "dq"):
        assert got[n].shape == q.shape and (got[n] == 0).all(), n
    assert np.isneginf(got["lse"]).all()


@pytest.mark.parametrize("D", [64, 128])
def test_no_queries(D):
    rng = np.random.default_rng(2401)
    none, k = np.zeros((0, 4, D), np.uint8), codes8(rng, (300, 2, D))
    got = run_attention(none, k, k, np.array([0, 0]), np.array([0, 300]), True, 0.125, none, max_q=8192)
    assert (got["dk"] == 0).all() and (got["dv"] == 0).all()
