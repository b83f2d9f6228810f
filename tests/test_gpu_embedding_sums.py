"""embed_bwd's sums are doubles, rounded once."""
import numpy as np
import pytest
import torch

import paper_1812_08011_amd as fp8t
from oracle import tokens as ot
from tests.gpu_util import DEV, dev, host, say
from tests.token_util import F32, draw, gpu, workspace  # noqa: F401

pytestmark = pytest.mark.gpu


def bwd(tok, e, V, scale):
    say(f"embed_bwd T={len(tok)} V={V} W={e.shape[1]} scale={scale}")
    td, ed, g = dev(tok), dev(e), torch.full((V, e.shape[1]), np.nan, device=DEV)
    n = fp8t.embed_bwd_workspace_size(td, ed, g)
    fp8t.embed_bwd(td, ed, g, scale, workspace(n), n)
    return host(g)


@pytest.mark.parametrize("W", [3, 24, 100, 260, 520])
@pytest.mark.parametrize("T", [1, 2, 17, 33, 100, 1000, 20000])
def test_small_errors_beside_large_ones(T, W):
    """Each row has as many errors of +2^30 as of -2^30 among small ones, in any
    order: doubles hold every sum of them, floats lose the small ones.  Runs in one
    share, over shares and over pieces."""
    rng = np.random.default_rng(170)
    tok = np.repeat(rng.permutation(np.minimum(rng.integers(0, 12, T), 9)), 3)
    e = (rng.integers(-63, 64, (3 * T, W)) / 64.0).astype(F32)
    e[0::3], e[2::3] = 2.0 ** 30, -2.0 ** 30
    order = rng.permutation(3 * T)
    tok, e = tok[order], e[order]
    want = np.zeros((13, W))
    np.add.at(want, tok, e.astype(np.float64))
    assert np.array_equal(bwd(tok, e, 13, 1.0), want.astype(F32))
    assert np.array_equal(bwd(tok, e, 13, 0.5), (want * 0.5).astype(F32))


def test_results_are_rounded_once():
    """n errors in doubles lose n 2^-53 of their magnitudes, the product with the
    scale 2^-53 of itself, the result 2^-24."""
    rng = np.random.default_rng(171)
    tok = np.minimum(rng.integers(0, 60, 9000), rng.integers(0, 60, 9000))
    e = draw(rng, (9000, 70), F32)
    scale = F32(3.7)
    want, bound = ot.embed_grad(tok, e.astype(np.float64), 60, float(scale))
    got = bwd(tok, e, 60, float(scale))
    assert (abs(got - want) <= abs(want) * 2.0 ** -24 + bound * 2.0 ** (24 - 52)).all()
    assert not (abs((e[tok == 0]).sum(0) * scale - want[0]) <= abs(want[0]) * 2.0 ** -24).all(), "floats do as well"
