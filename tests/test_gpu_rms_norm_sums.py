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
