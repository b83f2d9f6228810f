"""attn_fwd_fp8 and attn_bwd_fp8 under the plans that their size hints choose:
keys laid out in the workspace (many rows), keys shared out over workgroups
with partial results, few rows, queries shared out in dk and dv -- each at
lengths where it can go wrong, against the float64 definition; and replays of
a captured graph."""
import numpy as np
import pytest
import torch

import paper_1812_08011_amd as fp8t
from oracle import lm
from tests.gpu_util import DEV, dev, host, say
from tests.lm_util import offsets, run_attention, value
from tests.test_gpu_attention import INF8, LENS, NAN8, both, compare, operands

pytestmark = pytest.mark.gpu
MANY = 8192                                            # rows that a caller may expect per sequence


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    fp8t.lib()
    yield


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("D", [16, 64, 100, 128])
@pytest.mark.parametrize("lens", LENS, ids=str)
def test_lengths_with_keys_laid_out(lens, D, causal):
    both(1000 + D, *lens, 4, 2, D, causal, max_q=MANY)


@pytest.mark.parametrize("D", [1, 33, 65, 127, 128])
def test_strided_operands_with_keys_laid_out(D):
    both(1100 + D, [60, 1, 33], [60, 77, 33], 4, 2, D, True, strided=True, max_q=MANY)


@pytest.mark.parametrize("kw", [dict(max_q=MANY, max_k=MANY), dict(max_q=300, max_k=MANY),
                                dict(max_q=1, max_k=MANY)], ids=str)
@pytest.mark.parametrize("D", [64, 96])
def test_keys_shared_out(D, kw):
    """Key ranges that lie behind a row's last key, or behind every row's."""
    both(1200 + D, [70, 3, 0], [1500, 3, 40], 4, 1, D, True, **kw)
    both(1210 + D, [130], [1300], 2, 2, D, False, **kw)


@pytest.mark.parametrize("D", [64, 128])
def test_queries_shared_out(D):
    """Few keys under many queries: dk and dv from several query ranges."""
    both(1300 + D, [1500, 40], [90, 100], 4, 2, D, False)
    both(1310 + D, [1100], [1100], 2, 1, D, True)


@pytest.mark.parametrize("kw", [dict(max_q=MANY), dict(max_q=1), dict(max_q=300, max_k=MANY)], ids=str)
@pytest.mark.parametrize("bad", [NAN8, INF8])
@pytest.mark.parametrize("where", ["k", "v", "q", "e"])
def test_masked_places_do_not_enter(where, bad, kw):
    lens, at = [100, 75], 100 + 41
    q, k, v, e = operands(1400, lens, lens, 4, 2, 80)
    cu, c = offsets(lens), 0.125
    say(f"attention, {where}[{at}] = {bad:#x}, {kw}")
    clean = run_attention(q, k, v, cu, cu, True, c, e, **kw)
    ops = dict(q=q, k=k, v=v, e=e)
    ops[where] = ops[where].copy()
    ops[where][at] = bad
    got = run_attention(ops["q"], ops["k"], ops["v"], cu, cu, True, c, ops["e"], **kw)
    n = np.arange(175)
    keep_q = n < at if where in "kv" else n != at
    keep_fwd = np.ones(175, bool) if where == "e" else keep_q
    keep_k = n < 100 if where in "kv" else (n < 100) | (n > at)
    for name in ("o", "o8"):
        assert np.array_equal(got[name][keep_fwd], clean[name][keep_fwd]), name
    assert np.array_equal(got["lse"][:, keep_fwd], clean["lse"][:, keep_fwd])
    assert np.array_equal(got["dq"][keep_q], clean["dq"][keep_q])
    for name in ("dk", "dv"):
        assert np.array_equal(got[name][keep_k], clean[name][keep_k]), name
    assert not np.isfinite(value(got["dq"][at])).all()


@pytest.mark.parametrize("kw", [dict(max_q=MANY, max_k=200), dict(max_q=200, max_k=MANY),
                                dict(max_q=1, max_k=MANY)], ids=str)
def test_offsets_out_of_range_are_clamped(kw):
    say(f"attention with offsets outside the arrays, {kw}")
    q, k, v, e = operands(1500, [200], [200], 2, 2, 64)
    for cu in ([0, 200 + 10 ** 9], [-5, 200], [0, 140, 20, 10 ** 12], [-(10 ** 15), 10 ** 15]):
        run_attention(q, k, v, np.array(cu), np.array(cu), True, 0.125, e, **kw)
    cu = np.array([-3, 10 ** 9])
    got = run_attention(q, k, v, cu, cu, True, 0.125, e, **kw)
    ref = lm.attention(value(q), value(k), value(v), [0, 200], [0, 200], True, 0.125, value(e))
    compare(got, ref)


def test_replays_of_a_graph():
    """A captured forward and backward call, replayed between eager work."""
    say("attention in a graph")
    lens = [300, 0, 129]
    q, k, v, e = (dev(x) for x in operands(1600, lens, lens, 4, 1, 128))
    cu = dev(offsets(lens))
    args = (q, k, v, cu, cu, MANY, 300, True, 0.1)
    nf, nb = fp8t.attn_fwd_fp8_workspace_size(*args), fp8t.attn_bwd_fp8_workspace_size(*args)
    ws = torch.empty(max(nf, nb), dtype=torch.uint8, device=DEV)
    T = sum(lens)
    o = torch.zeros((T, 4, 128), dtype=torch.int16, device=DEV).view(torch.uint16)
    lse = torch.empty((4, T), dtype=torch.float32, device=DEV)
    grads = [torch.zeros((T, h, 128), dtype=torch.uint8, device=DEV) for h in (4, 1, 1)]
    outs = [o, lse, *grads]

    def run():
        fp8t.attn_fwd_fp8(*args, o, None, 1.0, lse, ws, nf)
        fp8t.attn_bwd_fp8(*args, o, e, lse, *grads, 1.0, ws, nb)

    def eager():
        run()
        torch.cuda.synchronize()
        return [host(x).copy() for x in outs]

    want = eager()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    other = torch.randint(0, 120, q.shape, dtype=torch.uint8, device=DEV)
    keep = q.clone()
    for i in range(3):
        ws.fill_(0xFF)
        q.copy_(other if i == 1 else keep)
        graph.replay()
        torch.cuda.synchronize()
        got = [host(x).copy() for x in outs]
        for a, b in zip(got, eager() if i == 1 else want):
            assert np.array_equal(a, b), i
