"""Attention's size hints (max_q, max_k) of any size choose a plan, and no more:
the workspace query answers for them as for the longest sequences there are."""
import os

import pytest

import paper_1812_08011_amd as fp8t

HUGE = [2 ** 31, 2 ** 40, 2 ** 60, 2 ** 61, 2 ** 62, 2 ** 63 - 1]


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(fp8t.LIB_PATH):
        pytest.skip("libfp8train.so is not built")
    return fp8t.lib()


@pytest.mark.parametrize("heads", [(1, 1), (8, 2), (12, 4), (16, 1)], ids=str)
@pytest.mark.parametrize("name", ["attn_fwd_fp8_workspace_size", "attn_bwd_fp8_workspace_size"])
def test_huge_hints(lib, name, heads):
    f, most = getattr(lib, name), (2 ** 31 - 4097) // (heads[0] // heads[1])
    for S, Tq, Tk in ((1, 5, 70000), (3, 4000, 900), (2, 1, 1)):
        want = f(S, Tq, Tk, most, 2 ** 31 - 4097, *heads, 128, 1)
        assert want > 0
        for n in HUGE:
            assert f(S, Tq, Tk, n, n, *heads, 128, 1) == want, (S, Tq, Tk, n)
            assert f(S, Tq, Tk, n, 2 ** 31 - 4097, *heads, 128, 1) == want, (S, Tq, Tk, n)
