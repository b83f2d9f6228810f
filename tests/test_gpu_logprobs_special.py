"""token_logprobs at values that the tests of its widths leave out."""
import numpy as np
import pytest
import torch

import paper_1812_08011_amd as fp8t
from oracle import tokens as ot
from tests.gpu_util import DEV, dev, host, say
from tests.lm_util import check, value
from tests.token_util import F16, F32, draw, gpu, workspace  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("k", [0, 7])
@pytest.mark.parametrize("V", [1, 60, 300, 2048, 3000, 9001, 20001, 70001])
@pytest.mark.parametrize("ty", [F32, F16])
def test_largest_logit_of_rows_that_are_not_finite(ty, V, k):
    """stats[n, 0] is the largest logit whatever it is: +Inf, -Inf, the type's
    largest, NaN where there is one; ln S is NaN of all but finite ones."""
    rng = np.random.default_rng(140)
    low, inf, nan, top = (-np.inf, np.inf, np.nan, F32(3.4028235e38)) if ty == F32 else (0xFE00, 0x7E00, 0x7F00, 0x7DFF)
    z = draw(rng, (9, V), ty, 2.0)
    z[1, V // 3] = inf
    z[2, V // 2] = nan
    z[3] = low
    z[4, V - 1], z[4, 0] = inf, nan
    z[5], z[5, V - 1] = low, inf
    z[6], z[6, 0] = low, nan
    z[7, V // 2] = top
    z[8] = inf
    want = ot.logprobs(value(z), np.zeros((9, 0), np.int64), 1.0, k)
    for rows in (slice(0, 9),) + tuple(slice(i, i + 1) for i in range(9)):
        zd = dev(z[rows])
        for n in sorted({0, fp8t.token_logprobs_workspace_size(zd, k)}):
            say(f"token_logprobs stats {rows} of {V} {ty.__name__} k={k} workspace={n}")
            stats = torch.full((len(zd), 2), 7.0, device=DEV)
            top_idx = torch.full((len(zd), k), -7, dtype=torch.int64, device=DEV) if k else None
            fp8t.token_logprobs(zd, None, 1.0, stats=stats, top_idx=top_idx, workspace=workspace(n), workspace_bytes=n)
            got = host(stats)
            assert np.array_equal(got[:, 0].astype(np.float64), want["stats"][rows, 0], equal_nan=True)
            check("ln S", got[:, 1], want["stats"][rows, 1], want["stats_err"][rows, 1])
            if k:
                assert np.array_equal(host(top_idx), want["top_idx"][rows])


@pytest.mark.parametrize("tau", [2.0, 4.0, 1e9])
@pytest.mark.parametrize("V", [5, 100, 3000, 70001])
def test_distances_past_the_range_of_floats(V, tau):
    """z - M beyond FP32's range, its quotient by tau within it: log probabilities
    of given tokens and of the likeliest ones are finite."""
    rng = np.random.default_rng(141)
    z = draw(rng, (4, V), F32)
    z[0], z[0, V // 2] = -3.2e38, 3.2e38
    z[1] = rng.uniform(-3.3e38, 3.3e38, V).astype(F32)
    z[2, 0], z[2, V - 1] = -3e38, 3e38
    idx = np.stack([rng.integers(0, V, 3) for _ in range(4)])
    idx[:, 0], idx[:, 1] = 0, V - 1
    want = ot.logprobs(value(z), idx, float(F32(tau)), 4)
    assert np.isfinite(want["logp"]).all()
    for rows in (slice(0, 4), slice(0, 1), slice(1, 2)):
        zd = dev(z[rows])
        for n in sorted({0, fp8t.token_logprobs_workspace_size(zd, 4)}):
            say(f"token_logprobs distances {rows} of {V} tau={tau} workspace={n}")
            nan = lambda *s: torch.full(s, np.nan, device=DEV)
            out = dict(logp=nan(len(zd), 3), entropy=nan(len(zd)), top_logp=nan(len(zd), 4))
            fp8t.token_logprobs(zd, dev(idx[rows]), tau, **out, workspace=workspace(n), workspace_bytes=n)
            for x in out:
                check(x, host(out[x]), want[x][rows], want[x + "_err"][rows])
