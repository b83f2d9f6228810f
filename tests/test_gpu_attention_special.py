"""Scores that are not numbers under every plan of attn_fwd_fp8: key
ranges shared out over workgroups and joined, one pass without a workspace,
keys laid out beforehand.  What a row sees decides its result, not the plan."""
import numpy as np
import pytest
import torch

import paper_1812_08011_amd as fp8t
from oracle import lm
from tests.gpu_util import say
from tests.lm_util import check, offsets, run_attention, value
from tests.test_gpu_attention import INF8, NAN8, operands

pytestmark = pytest.mark.gpu
MANY = 8192


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    fp8t.lib()
    yield


PLANS = [dict(), dict(workspace=False), dict(max_q=1, max_k=MANY), dict(max_q=300, max_k=MANY),
         dict(max_q=MANY), dict(max_q=MANY, max_k=MANY)]


def compare(q, k, v, cu_q, cu_k, causal, c, plans=PLANS):
    ref = lm.attention(value(q), value(k), value(v), cu_q, cu_k, causal, c)
    for kw in plans:
        say(f"  plan {kw}")
        got = run_attention(q, k, v, cu_q, cu_k, causal, c, **kw)
        check(f"lse {kw}", got["lse"], ref["lse"], ref["lse_err"])
        check(f"o {kw}", got["o"], ref["o"], ref["o_err"])
        check(f"o8 {kw}", got["o8"], ref["o"], ref["o_err"])


@pytest.mark.parametrize("bad", [NAN8, INF8, INF8 | 0x80])
@pytest.mark.parametrize("D,lens_k", [(64, [1024, 513]), (128, [512, 257]), (64, [1024, 1024]),
                                      (128, [300, 1])], ids=str)
def test_a_key_alone_in_its_range(D, lens_k, bad):
    """The newest key of one sequence, with ranges of eight tiles alone in the
    last of them, is not finite: its row is not, the other sequence's is."""
    say(f"attention, newest key {bad:#x}, D={D}, {lens_k}")
    q, k, v, _ = operands(2000 + D, [1, 1], lens_k, 1, 1, D)
    k[-1] = bad
    compare(q, k, v, offsets([1, 1]), offsets(lens_k), True, 0.125)


@pytest.mark.parametrize("D", [64, 100, 128])
def test_a_query_that_is_not_a_number(D):
    """Every score is NaN: so are o and lse (-Inf says that a row sees no key)."""
    say(f"attention, a NaN query, D={D}")
    lens_q, lens_k = [2, 40], [2000, 700]
    q, k, v, _ = operands(2100 + D, lens_q, lens_k, 4, 2, D)
    q[1, 2], q[30, 0] = NAN8, NAN8
    compare(q, k, v, offsets(lens_q), offsets(lens_k), True, 0.125)


@pytest.mark.parametrize("D", [64, 128])
def test_every_visible_score_of_a_range_is_not_a_number(D):
    """All keys of the first or of the last ranges."""
    say(f"attention, ranges of NaN keys, D={D}")
    lens_q, lens_k = [1, 1, 1], [2048, 2048, 2048]
    q, k, v, _ = operands(2200 + D, lens_q, lens_k, 2, 1, D)
    k[:1024] = NAN8
    k[4096 - 600:4096] = NAN8
    compare(q, k, v, offsets(lens_q), offsets(lens_k), True, 0.125)
