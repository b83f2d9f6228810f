"""attn_fwd_fp8 and attn_bwd_fp8 against the float64 definition (oracle/lm.py),
within the bounds that it derives: lengths from zero to long, odd head
dimensions, grouped heads, strided operands, rows that see nothing, values
that are not finite in masked places, long histories and wide offsets."""
import numpy as np
import pytest
import torch

import oracle
import paper_1812_08011_amd as fp8t
from oracle import lm
from tests.gpu_util import DEV, dev, host, say
from tests.lm_util import check, codes8, offsets, run_attention, value

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    fp8t.lib()
    yield


def operands(seed, lens_q, lens_k, Hq, Hkv, D, std=1.0):
    rng = np.random.default_rng(seed)
    Tq, Tk = sum(lens_q), sum(lens_k)
    return [codes8(rng, (n, h, D), std) for n, h in ((Tq, Hq), (Tk, Hkv), (Tk, Hkv), (Tq, Hq))]


def compare(got, ref, scales=(1.0, 1.0)):
    check("lse", got["lse"], ref["lse"], ref["lse_err"])
    check("o", got["o"], ref["o"], ref["o_err"])
    # FP8: the rounding of the FP32 value; the scales here are powers of two
    check("o8", got["o8"], ref["o"] * scales[0], ref["o_err"] * scales[0])
    for n in ("dq", "dk", "dv"):
        if n in got:
            check(n, got[n], ref[n] * scales[1], ref[n + "_err"] * scales[1])


def both(seed, lens_q, lens_k, Hq, Hkv, D, causal, grad=np.uint16, scales=(1.0, 1.0), std=1.0, **kw):
    say(f"attention {lens_q} over {lens_k} Hq={Hq} Hkv={Hkv} D={D} causal={causal} {kw}")
    q, k, v, e = operands(seed, lens_q, lens_k, Hq, Hkv, D, std)
    cu_q, cu_k, c = offsets(lens_q), offsets(lens_k), 1.0 / np.sqrt(D)
    c = float(np.float32(c))
    got = run_attention(q, k, v, cu_q, cu_k, causal, c, e, grad, scales, **kw)
    ref = lm.attention(value(q), value(k), value(v), cu_q, cu_k, causal, c, value(e))
    compare(got, ref, scales)
    return got


LENS = [
    ([1], [1]),
    ([1, 1, 1], [1, 2, 200]),
    ([2, 31, 32, 33], [2, 31, 32, 33]),
    ([64, 0, 65, 1], [64, 5, 65, 0]),                 # no queries; no keys
    ([130, 7], [130, 7]),
    ([5, 40], [300, 41]),                             # new tokens over a history
    ([70, 9], [40, 9]),                               # more queries than keys: rows that see none
]


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("D", [16, 64, 80, 128])
@pytest.mark.parametrize("lens", LENS, ids=str)
def test_lengths(lens, D, causal):
    both(100 + D, *lens, 4, 2, D, causal)


@pytest.mark.parametrize("D", [1, 2, 3, 31, 33, 63, 65, 100, 127])
def test_odd_head_dimensions(D):
    both(200 + D, [45, 3], [45, 80], 2, 1, D, True)


@pytest.mark.parametrize("heads", [(1, 1), (5, 5), (6, 3), (8, 1), (7, 1), (40, 1), (12, 4)], ids=str)
@pytest.mark.parametrize("lens", [([50, 2], [50, 90]), ([1, 1], [170, 3])], ids=str)
def test_grouped_heads(heads, lens):
    both(300 + heads[0], *lens, *heads, 64, True)


@pytest.mark.parametrize("D", [64, 100, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_strided_operands_and_results(D, causal):
    """Slices of wider buffers at odd addresses, NaN around the operands."""
    both(400 + D, [60, 1, 33], [60, 77, 33], 4, 2, D, causal, strided=True)


@pytest.mark.parametrize("grad", [np.uint8, np.uint16])
def test_scales_and_gradient_formats(grad):
    both(500, [40, 90], [40, 90], 4, 2, 64, True, grad, (8.0, 0.25))


def test_sharp_and_large_scores():
    """Scores in the thousands: one key takes each row."""
    both(600, [70], [70], 2, 2, 64, True, std=8.0)


def test_heads_outside_tokens():
    """H x T x D storage: the head stride above the token stride."""
    say("attention with H x T x D storage")
    q, k, v, e = operands(700, [90], [90], 4, 2, 64)
    cu, c = offsets([90]), 0.125
    turned = lambda a: dev(np.ascontiguousarray(a.transpose(1, 0, 2))).transpose(0, 1)
    args = (turned(q), turned(k), turned(v), dev(cu), dev(cu), 90, 90, True, c)
    o = torch.zeros((4, 90, 64), dtype=torch.uint8, device=DEV).to(torch.uint16).transpose(0, 1)
    lse = torch.empty((4, 90), dtype=torch.float32, device=DEV)
    fp8t.attn_fwd_fp8(*args, o, None, 1.0, lse)
    n = fp8t.attn_bwd_fp8_workspace_size(*args)
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    grads = [torch.zeros((h, 90, 64), dtype=torch.uint8, device=DEV).transpose(0, 1) for h in (4, 2, 2)]
    fp8t.attn_bwd_fp8(*args, o, turned(e), lse, *grads, 1.0, ws, n)
    ref = lm.attention(value(q), value(k), value(v), cu, cu, True, c, value(e))
    check("o", host(o.contiguous()), ref["o"], ref["o_err"])
    for name, g in zip(("dq", "dk", "dv"), grads):
        check(name, host(g.contiguous()), ref[name], ref[name + "_err"])


def test_shared_keys_by_a_zero_stride():
    """One key/value row broadcast over the tokens (token stride 0)."""
    say("attention with a broadcast key")
    q, k, v, _ = operands(710, [20], [1], 2, 2, 32)
    cu = dev(offsets([20]))
    lse = torch.empty((2, 20), dtype=torch.float32, device=DEV)
    o8 = torch.empty((20, 2, 32), dtype=torch.uint8, device=DEV)
    fp8t.attn_fwd_fp8(dev(q), dev(k).expand(20, 2, 32), dev(v).expand(20, 2, 32), cu, cu, 20, 20,
                      False, 0.5, None, o8, 1.0, lse)
    assert np.array_equal(host(o8), np.broadcast_to(v, (20, 2, 32)))


NAN8, INF8 = 0x7F, 0x7C


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("bad", [NAN8, INF8])
@pytest.mark.parametrize("where", ["k", "v", "q", "e"])
def test_masked_places_do_not_enter(where, bad, D):
    """Causal, one token of the sequence not finite: rows that do not see it
    are what they are without it."""
    lens, at = [100, 75], 100 + 41                        # token 41 of the second sequence
    q, k, v, e = operands(800, lens, lens, 4, 2, D)
    cu, c = offsets(lens), 0.125
    say(f"attention, {where}[{at}] = {bad:#x}, D={D}")
    clean = run_attention(q, k, v, cu, cu, True, c, e)
    ops = dict(q=q, k=k, v=v, e=e)
    ops[where] = ops[where].copy()
    ops[where][at] = bad
    got = run_attention(ops["q"], ops["k"], ops["v"], cu, cu, True, c, ops["e"])
    first = np.arange(175) < 100                          # the other sequence
    before = np.arange(175) < at                          # queries that do not see the token
    after = np.arange(175) > at                           # keys that the token does not see
    keep_q = before if where in "kv" else np.arange(175) != at
    if where == "e":
        keep_fwd = np.ones(175, bool)
    else:
        keep_fwd = keep_q
    for n in ("o", "o8"):
        assert np.array_equal(got[n][keep_fwd], clean[n][keep_fwd]), n
    assert np.array_equal(got["lse"][:, keep_fwd], clean["lse"][:, keep_fwd])
    assert np.array_equal(got["dq"][keep_q], clean["dq"][keep_q])
    keep_k = first if where in "kv" else first | after
    for n in ("dk", "dv"):
        assert np.array_equal(got[n][keep_k], clean[n][keep_k]), n
    # and what sees it is not finite
    if where != "e":
        assert np.isnan(value(got["o"][at])).any() or bad == INF8
    assert not np.isfinite(value(got["dq"][at])).all()


def test_a_long_history_is_shared_out():
    """Few rows over long histories: the plan with partial results and the one
    without agree with the definition."""
    rng = np.random.default_rng(900)
    lens_q, lens_k, Hq, Hkv, D = [1, 2, 1], [5000, 3001, 7], 4, 2, 64
    q, k, v, _ = operands(900, lens_q, lens_k, Hq, Hkv, D)
    cu_q, cu_k, c = offsets(lens_q), offsets(lens_k), 0.125
    ref = lm.attention(value(q), value(k), value(v), cu_q, cu_k, True, c)
    for kw in (dict(), dict(workspace=False), dict(max_q=1, max_k=1), dict(max_k=10 ** 6)):
        say(f"attention, long history, {kw}")
        compare(run_attention(q, k, v, cu_q, cu_k, True, c, **kw), ref)
    # a far key that is not finite stays out of the rows that do not see it
    k2, v2 = k.copy(), v.copy()
    k2[cu_k[2] - 1], v2[cu_k[2] - 1] = NAN8, NAN8           # seen by the second of two rows only
    got = run_attention(q, k2, v2, cu_q, cu_k, True, c)
    want = run_attention(q, k, v, cu_q, cu_k, True, c)
    for t in (0, 1, 3):
        assert np.array_equal(got["o"][t], want["o"][t]), t
    assert np.isnan(value(got["o"][2])).all()


def test_offsets_past_32_bits():
    """Keys and values 2^32 bytes into their buffers."""
    D, stride = 64, 65536
    Tk, n = 70000, 300
    say("attention past 2^32 bytes")
    rng = np.random.default_rng(910)
    kb = torch.empty((Tk * stride,), dtype=torch.uint8, device=DEV)
    kv = kb.as_strided((Tk, 2, D), (stride, D, 1))
    k, v, q = codes8(rng, (n, 1, D)), codes8(rng, (n, 1, D)), codes8(rng, (5, 1, D))
    kv[Tk - n:, 0:1] = dev(k)
    kv[Tk - n:, 1:2] = dev(v)
    cu_q, cu_k = np.array([0, 0, 5]), np.array([0, Tk - n, Tk])
    o = torch.empty((5, 1, D), dtype=torch.uint16, device=DEV)
    lse = torch.empty((1, 5), dtype=torch.float32, device=DEV)
    fp8t.attn_fwd_fp8(dev(q), kv[:, 0:1], kv[:, 1:2], dev(cu_q), dev(cu_k), 5, n, True, 0.125, o,
                      None, 1.0, lse)
    ref = lm.attention(value(q), value(k), value(v), [0, 5], [0, n], True, 0.125)
    check("o", host(o), ref["o"], ref["o_err"])
    check("lse", host(lse), ref["lse"], ref["lse_err"])


def test_offsets_out_of_range_are_clamped():
    """Offsets outside the arrays and decreasing ones stay inside them."""
    say("attention with offsets outside the arrays")
    q, k, v, e = operands(920, [64], [64], 2, 2, 64)
    for cu in ([0, 64 + 10 ** 9], [-5, 64], [0, 40, 20, 10 ** 12], [-(10 ** 15), 10 ** 15]):
        run_attention(q, k, v, np.array(cu), np.array(cu), True, 0.125, e, max_q=64, max_k=64)
    ref = lm.attention(value(q), value(k), value(v), [0, 64], [0, 64], True, 0.125)
    got = run_attention(q, k, v, np.array([-3, 10 ** 9]), np.array([-7, 10 ** 9]), True, 0.125,
                        max_q=64, max_k=64)
    check("o", got["o"], ref["o"], ref["o_err"])


def test_optional_results_and_nothing_to_do():
    say("attention, optional results")
    q, k, v, _ = operands(930, [30], [30], 2, 2, 32)
    cu = dev(offsets([30]))
    args = (dev(q), dev(k), dev(v), cu, cu, 30, 30, True, 0.2)
    o = torch.empty((30, 2, 32), dtype=torch.uint16, device=DEV)
    o8 = torch.empty((30, 2, 32), dtype=torch.uint8, device=DEV)
    lse = torch.empty((2, 30), dtype=torch.float32, device=DEV)
    fp8t.attn_fwd_fp8(*args, o, o8, 1.0, lse)
    for pick in range(3):
        alone = [torch.zeros_like(x) if i == pick else None for i, x in enumerate((o.view(torch.int16),
                                                                                o8, lse))]
        fp8t.attn_fwd_fp8(*args, None if alone[0] is None else alone[0].view(torch.uint16), alone[1],
                          1.0, alone[2])
        same = (o.view(torch.int16), o8, lse)[pick]
        assert torch.equal(alone[pick], same)
    with pytest.raises(fp8t.Fp8tError):
        fp8t.attn_fwd_fp8(*args, None, None)
    none = lambda h: torch.empty((0, h, 32), dtype=torch.uint8, device=DEV)
    zero = torch.zeros(1, dtype=torch.int64, device=DEV)
    fp8t.attn_fwd_fp8(none(2), none(2), none(2), zero, zero, 0, 0, True, 0.2,
                      None, none(2), 1.0, None)


def test_runs_repeat_and_streams_are_kept():
    """The same bits on every run, and on a stream of the caller's."""
    lens = [300, 64, 129]
    q, k, v, e = operands(940, lens, lens, 4, 1, 128)
    say("attention on another stream")
    a = run_attention(q, k, v, offsets(lens), offsets(lens), True, 0.1, e)
    side = torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(side):
            b = run_attention(q, k, v, offsets(lens), offsets(lens), True, 0.1, e)
        for n in a:
            assert np.array_equal(a[n], b[n]), n


def test_longer_sequences():
    """Several tiles of queries and keys, grouped heads, both directions."""
    both(950, [513, 260], [513, 260], 2, 1, 128, True)
    both(951, [300], [700], 3, 3, 64, False)
