"""rms_norm_bwd's long sums: terms that cancel, which sums in floats would lose."""
import numpy as np
import pytest
import torch

import paper_1812_08011_amd as fp8t
from tests.gpu_util import DEV, dev, host, say
from tests.lm_util import value
from tests.token_util import F8, F16, F32, TORCH, draw, gpu, rounded, workspace  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,W", [(8192, 40), (8192, 600), (4096, 1500), (4096, 4096), (2048, 8192), (2048, 8200), (4096, 9001),
                                 (2048, 16384), (2048, 20000)])
def test_weight_gradient_keeps_small_terms(T, W):
    """Columns of +2^22, a small number, -2^22 and a small number in turn; all
    products are exact.  A workgroup's rows are whole turns, so that its sum has
    24 bits and doubles give the total of the small ones; a float beside 2^22
    has a step of 1/2 and loses them all."""
    parts = fp8t.rms_norm_bwd_workspace_size(torch.empty((T, W), dtype=torch.uint8)) // (4 * W)
    assert T % parts == 0 and T // parts % 4 == 0, "whole turns"
    rng = np.random.default_rng(130)
    turns = rng.integers(-31, 32, (T, 8)) / 64.0
    turns[0::4], turns[2::4] = 2.0 ** 22, -2.0 ** 22
    h = np.tile(rounded(turns, F16), (1, -(-W // 8)))[:, :W]
    want = np.tile(turns.sum(0), -(-W // 8))[:W]
    for dy, ty in ((0x3C, F8), (31 << 9, F16)):                 # 1
        say(f"rms_norm_bwd {T}x{W} sums of {T // parts} rows, dy {ty.__name__}")
        dw, hd = torch.full((W,), np.nan, device=DEV), dev(h)
        n = fp8t.rms_norm_bwd_workspace_size(hd)
        fp8t.rms_norm_bwd(hd, None, torch.ones(T, device=DEV), dev(np.full((T, W), dy, ty)), None, None, None, 1.0, dw,
                          workspace(n), n)
        assert np.array_equal(host(dw), want.astype(F32))
        # with the rows' own gradients formed on the way
        again, dx = torch.full((W,), np.nan, device=DEV), torch.empty((T, W), dtype=torch.uint16, device=DEV)
        fp8t.rms_norm_bwd(hd, None, torch.ones(T, device=DEV), dev(np.full((T, W), dy, ty)), None, dx, None, 1.0, again,
                          workspace(n), n)
        assert np.array_equal(host(again), host(dw))


@pytest.mark.parametrize("W", [7, 64, 100, 200, 500, 1000, 2048, 4096, 8192, 8200, 16384, 20003])
def test_row_mean_keeps_small_terms(W):
    """Four rows whose small products stand beside +2^24 and -2^24, and random ones.
    From a mean rounded once the gradient follows in float products: bit for bit in
    random rows.  In the first ones an addition of doubles next to 2^24 loses 2^-29,
    so that two orders' means are 2^-28 apart before they are rounded (2^-24 of
    themselves each) and n m, g - n m and the residual's sum by their roundings; a
    float there loses 1 with every addition."""
    rng = np.random.default_rng(131)
    T = 12
    h, dy, dr = draw(rng, (T, W), F32), draw(rng, (T, W), F16), draw(rng, (T, W), F32)
    w, rstd = draw(rng, W, F32), np.exp(rng.standard_normal(T)).astype(F32)
    h[:4], rstd[:4] = rng.integers(-31, 32, (4, W)) / F32(64), 1
    for row in range(4):
        at = rng.permutation(W)[:2]
        h[row, at] = 2.0 ** 24, -2.0 ** 24
        w[at], dy[row, at] = 1, 31 << 9
    for r in (None, dr):
        say(f"rms_norm_bwd {T}x{W} mean, residual {r is not None}")
        dx, dx8 = torch.empty((T, W), device=DEV), torch.empty((T, W), dtype=torch.uint8, device=DEV)
        fp8t.rms_norm_bwd(dev(h), dev(w), dev(rstd), dev(dy), None if r is None else dev(r), dx, dx8, 4.0)
        n, g = h * rstd[:, None], value(dy).astype(F32) * w
        m = ((g * n).astype(np.float64).sum(1) / W).astype(F32)
        own = rstd[:, None] * (g - n * m[:, None])
        d = own if r is None else r + own
        got = host(dx)
        assert np.array_equal(got[4:], d[4:])
        f = lambda a: abs(a[:4].astype(np.float64))
        nm = f(n) * f(m[:, None])
        lim = f(n) * 2.0 ** -28 + 2.0 ** -23 * (3 * nm + f(g) + f(d))
        assert (f(got - d.astype(np.float64)) <= lim).all(), np.argwhere(f(got - d.astype(np.float64)) > lim)[:5]
        assert np.array_equal(host(dx8), rounded(got, F8, 4.0))
