"""Result strides whose products pass 64 bits are checked like any others."""
import os

import pytest

import paper_1812_08011_amd as fp8t
from tests.test_lm_abi import FAKE, attn_args

E = fp8t.EINVAL


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(fp8t.LIB_PATH):
        pytest.skip("libfp8train.so is not built")
    return fp8t.lib()


@pytest.mark.parametrize("ts,hs", [(2 ** 62, 2 ** 62), (2 ** 62 + 64, 2 ** 62), (2 ** 62, 2 ** 62 + 63)])
def test_rows_that_overlap(lib, ts, hs):
    """Strides so near each other that row (1, 0) lies in row (0, 1)."""
    assert lib.rotary_embed(FAKE, 1, 192, 64, FAKE, FAKE, 3, 3, 65, 0, 0, 0, 1.0, 1.0, FAKE, 2, ts, hs,
                            None) == E
    three = dict(Tq=3, Tk=3, Hq=3, Hkv=3, D=65, qts=195, qhs=65, kts=195, khs=65, vts=195, vhs=65, ots=195,
                 ohs=65, o8ts=195, o8hs=65)
    assert lib.attn_fwd_fp8(*attn_args(False, **{**three, "ots": ts, "ohs": hs})) == E
    assert lib.attn_bwd_fp8(*attn_args(True, **{**three, "ets": 195, "ehs": 65, "dkts": 195, "dkhs": 65,
                                                "dvts": 195, "dvhs": 65, "dqts": ts, "dqhs": hs, "ws": FAKE,
                                                "wsb": 1 << 30})) == E
