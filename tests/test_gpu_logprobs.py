"""token_logprobs and token_logprobs_bwd against the float64 definitions
(oracle/tokens.py) within the bounds that they derive; the likeliest tokens are
whole numbers and equal."""
import numpy as np
import pytest
import torch

import paper_1812_08011_amd as fp8t
from oracle import tokens as ot
from tests.gpu_util import DEV, dev, host, say
from tests.lm_util import check, value
from tests.token_util import F8, F16, F32, Wide, draw, gpu, replayed, workspace  # noqa: F401

pytestmark = pytest.mark.gpu
NAMES = ("logp", "entropy", "stats", "top_idx", "top_logp")


def given(rng, N, V, m):
    idx = rng.integers(0, V, (N, m))
    return np.where(rng.random((N, m)) < 0.15, rng.choice([-1, V, 2 ** 40], (N, m)), idx)


def run(z, idx, tau, k, use_ws, pad=0, shift=0, want=NAMES):
    N, V = z.shape
    m = idx.shape[1]
    zd = Wide(N, V, z.dtype.type, pad, shift, z).view
    nan = lambda *s: torch.full(s, np.nan, device=DEV)
    out = dict(logp=nan(N, m), entropy=nan(N), stats=nan(N, 2),
               top_idx=torch.full((N, k), -7, dtype=torch.int64, device=DEV), top_logp=nan(N, k))
    n = fp8t.token_logprobs_workspace_size(zd, k) if use_ws else 0
    fp8t.token_logprobs(zd, dev(idx), tau, **{x: out[x] if x in want else None for x in NAMES},
                        workspace=workspace(n), workspace_bytes=n)
    return {x: host(out[x]) for x in want}


def compare(z, idx, tau, k, **kw):
    want = ot.logprobs(value(z), idx, float(np.float32(tau)), k)
    for use_ws in (True, False):
        say(f"logprobs {z.shape} {z.dtype} m={idx.shape[1]} k={k} tau={tau} ws={use_ws} {kw}")
        got = run(z, idx, tau, k, use_ws, **kw)
        assert np.array_equal(got["top_idx"], want["top_idx"]), np.argwhere(got["top_idx"] != want["top_idx"])[:5]
        for n in ("logp", "entropy", "top_logp"):
            check(n, got[n], want[n], want[n + "_err"])
        # the largest of a row that has none to speak of is not looked at
        fine = np.isfinite(want["stats"][:, 1])
        check("stats", got["stats"][fine], want["stats"][fine], want["stats_err"][fine])
        assert np.isnan(got["stats"][~fine, 1]).all()
    return got


@pytest.mark.parametrize("ty", [F32, F16])
@pytest.mark.parametrize("V", [1, 2, 7, 8, 9, 63, 255, 256, 2047, 2048, 2049, 6000, 16384, 16391, 40000, 70001])
def test_widths(V, ty):
    rng = np.random.default_rng(80)
    for N, k in ((3, 5), (1, 20)):
        compare(draw(rng, (N, V), ty, 2.0), given(rng, N, V, 2), 1.0, k)


@pytest.mark.parametrize("V", [131072, 300007, 1000003])
def test_wide_rows(V):
    rng = np.random.default_rng(81)
    compare(draw(rng, (2, V), F16, 2.0), given(rng, 2, V, 3), 0.7, 64)
    compare(draw(rng, (1, V), F32, 2.0), given(rng, 1, V, 3), 2.0, 128)


@pytest.mark.parametrize("k", [0, 1, 2, 63, 64, 65, 100, 128])
@pytest.mark.parametrize("V", [50, 129, 3000, 30000])
def test_top_counts(V, k):
    rng = np.random.default_rng(82)
    compare(draw(rng, (4, V), F16), given(rng, 4, V, 1), 1.0, k)
    compare(draw(rng, (2, V), F32), given(rng, 2, V, 0), 1.0, k)


@pytest.mark.parametrize("pad,shift", [(0, 1), (5, 0), (3, 2)])
@pytest.mark.parametrize("ty", [F32, F16])
def test_row_strides_and_addresses(pad, shift, ty):
    rng = np.random.default_rng(83)
    for V in (100, 9001, 33001):
        compare(draw(rng, (3, V), ty), given(rng, 3, V, 2), 1.0, 9, pad=pad, shift=shift)


@pytest.mark.parametrize("V", [300, 5000, 20001, 150001])
def test_ties_and_orders(V):
    """Rows of equal logits, of few different ones, ascending and descending
    ones, and the largest all beside each other."""
    rng = np.random.default_rng(84)
    z = np.zeros((8, V), F32)
    z[1] = rng.integers(0, 3, V)
    z[2] = np.linspace(-5, 5, V)
    z[3] = z[2][::-1]
    z[4] = rng.standard_normal(V)
    z[4, V // 3:V // 3 + 200] += 10
    z[5] = np.where(rng.random(V) < 0.5, 0.0, -0.0)
    z[6] = -3e38
    z[6, V - 2:] = 1.0
    z[7, ::8] = 1.0                                            # all of them first of eight
    for k in (1, 7, 128):
        compare(z, given(rng, 8, V, 1), 1.0, k)
        compare(z[:1], given(rng, 1, V, 1), 1.0, k)


@pytest.mark.parametrize("V", [200, 9000, 60001])
def test_masks_and_rows_that_are_not_finite(V):
    rng = np.random.default_rng(85)
    for ty in (F32, F16):
        z = draw(rng, (9, V), ty, 2.0)
        low, inf, nan = (F32(-np.inf), F32(np.inf), F32(np.nan)) if ty == F32 else (0xFE00, 0x7E00, 0x7F00)
        clean = compare(z, np.tile([[3, V - 1]], (9, 1)), 1.0, 20)
        z[1, rng.random(V) < 0.6] = low
        z[2] = low
        z[3], z[3, V // 2] = low, z[0, 0]
        z[4, V // 3] = inf
        z[5, V // 5] = nan
        z[6], z[6, 9] = low, nan
        z[7, 4:] = low                                         # fewer than k
        idx = np.tile([[3, V - 1]], (9, 1))
        got = compare(z, idx, 1.0, 20)
        for n in NAMES:
            assert np.array_equal(got[n][[0, 8]], clean[n][[0, 8]])
        compare(z[2:3], idx[:1], 1.0, 20)
        compare(z[5:6], idx[:1], 1.0, 20)


def test_large_logits():
    rng = np.random.default_rng(86)
    z = draw(rng, (4, 3000), F32, 1e4)
    z[1] += F32(1e7)
    z[2] *= F32(1e30)
    z[3] = np.where(rng.random(3000) < 0.5, F32(-1.5e38), F32(1.5e38))
    compare(z, given(rng, 4, 3000, 2), 1.0, 8)
    compare(draw(rng, (2, 3000), F16, 1e4), given(rng, 2, 3000, 2), 4.0, 8)


def test_one_result_at_a_time():
    rng = np.random.default_rng(87)
    for N, V in ((3, 700), (2, 60000)):
        z, idx = draw(rng, (N, V), F16), given(rng, N, V, 2)
        want = run(z, idx, 1.0, 6, True)
        for n in NAMES:
            assert np.array_equal(run(z, idx, 1.0, 6, True, want=(n,))[n], want[n]), n


def test_many_rows_and_given_tokens():
    rng = np.random.default_rng(88)
    compare(draw(rng, (1500, 300), F16), given(rng, 1500, 300, 2), 1.0, 4)
    compare(draw(rng, (2, 900), F16), given(rng, 2, 900, 4096), 1.0, 4)
    run(np.zeros((0, 5), F32), np.zeros((0, 2), np.int64), 1.0, 3, True)


def test_entries_for_a_distillation():
    """The top of a teacher's logits given to distill_loss: the teacher itself
    as the student of its own full top has no loss but its rounding."""
    rng = np.random.default_rng(89)
    z = draw(rng, (5, 100), F32)
    got = run(z, np.zeros((5, 0), np.int64), 1.0, 128, True, want=("top_idx", "top_logp"))
    loss = torch.empty(5, device=DEV)
    fp8t.distill_loss(dev(z), dev(got["top_idx"]), dev(got["top_logp"]), None, 2.0, 1.0, loss, None)
    assert (abs(host(loss)) <= 4 * 100 * 2.0 ** -22).all()


# ---- gradient --------------------------------------------------------------------------


def forward(z, idx, tau):
    r = ot.logprobs(value(z), idx, float(np.float32(tau)), 0)
    return r["stats"].astype(F32), r["entropy"].astype(F32)


def grad(z, idx, tau, stats, H, dl, dh, scale, ty, pad=0, shift=0):
    N, V = z.shape
    zd, g = Wide(N, V, z.dtype.type, pad, shift, z), Wide(N, V, ty, pad, shift)
    put = lambda a: None if a is None else dev(a)
    fp8t.token_logprobs_bwd(zd.view, dev(idx), tau, dev(stats), put(H), put(dl), put(dh), scale, g.view)
    return g.result()


def compare_grad(z, idx, tau, dl, dh, scale, ty, **kw):
    say(f"logprobs_bwd {z.shape} {z.dtype} m={idx.shape[1]} -> {ty.__name__} {dl is not None} "
        f"{dh is not None} {kw}")
    stats, H = forward(z, idx, tau)
    got = grad(z, idx, tau, stats, None if dh is None else H, dl, dh, scale, ty, **kw)
    f = lambda a: None if a is None else a.astype(np.float64)
    want, err = ot.logprobs_grad(value(z), idx, float(np.float32(tau)), f(stats), f(H), f(dl), f(dh),
                                 float(np.float32(scale)))
    check("g", got, want, err)
    return got


@pytest.mark.parametrize("g", [F32, F16, F8])
@pytest.mark.parametrize("ty", [F32, F16])
def test_gradient_formats(ty, g):
    rng = np.random.default_rng(90)
    N, V = 6, 777
    z, idx = draw(rng, (N, V), ty, 2.0), given(rng, N, V, 3)
    dl, dh = draw(rng, (N, 3), F32), draw(rng, N, F32)
    compare_grad(z, idx, 1.0, dl, dh, 64.0, g)
    compare_grad(z, idx, 2.0, dl, None, 64.0, g)
    compare_grad(z, idx[:, :0], 0.7, None, dh, 64.0, g)


@pytest.mark.parametrize("V", [1, 2, 7, 8, 9, 2048, 8191, 8192, 8193, 20001, 70001])
@pytest.mark.parametrize("ty", [F32, F16])
def test_gradient_widths_and_addresses(V, ty):
    rng = np.random.default_rng(91)
    z, idx = draw(rng, (3, V), ty), given(rng, 3, V, 2)
    dl, dh = draw(rng, (3, 2), F32), draw(rng, 3, F32)
    compare_grad(z, idx, 1.0, dl, dh, 8.0, ty)
    compare_grad(z, idx, 1.0, dl, dh, 8.0, F8, pad=3, shift=1)


@pytest.mark.parametrize("m", [1, 5, 64, 300, 4096])
def test_gradient_of_given_tokens(m):
    """Every place of a chunk and its borders; the same token many times."""
    rng = np.random.default_rng(92)
    V = 17000
    idx = given(rng, 3, V, m)
    idx[0] = rng.choice([0, 7, 8, 8191, 8192, 8193, 16383, 16384, V - 1], m)
    idx[1] = 8192
    compare_grad(draw(rng, (3, V), F16), idx, 1.0, draw(rng, (3, m), F32), None, 1.0, F32)


def test_gradient_rows_without_weight():
    """All gradients 0, or of unused entries only: +0 whatever the logits hold;
    unused entries' gradients are not looked at."""
    rng = np.random.default_rng(93)
    z, idx = draw(rng, (6, 500), F32), given(rng, 6, 500, 2)
    dl, dh = draw(rng, (6, 2), F32), draw(rng, 6, F32)
    idx[:] = rng.integers(0, 500, (6, 2))
    stats, H = forward(z, idx, 1.0)
    z[0, 5], dl[0], dh[0] = np.nan, 0, 0
    z[1, 5], idx[1], dh[1] = np.inf, [-1, 500], 0
    stats[1] = np.nan
    dl[2, 1], idx[2, 1] = np.nan, -1
    for ty in (F32, F16, F8):
        say("logprobs_bwd rows without weight")
        g = grad(z, idx, 1.0, stats, H, dl, dh, 2.0, ty)
        assert (value(g[:2]) == 0).all() and not np.signbit(value(g[:2])).any()
        f = lambda a: a.astype(np.float64)
        want, err = ot.logprobs_grad(f(z[2:]), idx[2:], 1.0, f(stats[2:]), f(H[2:]), f(dl[2:]), f(dh[2:]), 2.0)
        check("g", g[2:], want, err)


def test_gradient_of_masked_logits():
    rng = np.random.default_rng(94)
    z, idx = draw(rng, (4, 9000), F32), rng.integers(0, 9000, (4, 2))
    z[0, rng.random(9000) < 0.5] = -np.inf
    z[1] = -3e38
    z[1, idx[1, 0]] = 0.0
    z[2, idx[2, 0]] = -np.inf                                   # a given token that is masked
    z[3] = -np.inf
    dl, dh = draw(rng, (4, 2), F32), draw(rng, 4, F32)
    stats, H = forward(z, idx, 1.0)
    assert np.isfinite(grad(z, idx, 1.0, stats, H, dl, dh, 1.0, F32)[:3]).all()
    compare_grad(z[:3], idx[:3], 1.0, dl[:3], dh[:3], 1.0, F32)
    assert np.isnan(grad(z, idx, 1.0, stats, H, dl, dh, 1.0, F32)[3]).all()


def test_gradient_in_place():
    rng = np.random.default_rng(95)
    for ty in (F32, F16):
        for V in (600, 20001):
            say("logprobs_bwd in place")
            z, idx, dl = draw(rng, (4, V), ty), given(rng, 4, V, 3), draw(rng, (4, 3), F32)
            stats, H = forward(z, idx, 1.0)
            want = grad(z, idx, 1.0, stats, H, dl, H, 1.0, ty)
            zd = dev(z)
            fp8t.token_logprobs_bwd(zd, dev(idx), 1.0, dev(stats), dev(H), dev(dl), dev(H), 1.0, zd)
            assert np.array_equal(host(zd), want)


def test_gradient_is_the_difference_quotient():
    """Central differences of the FP32 results, step 2^-4: truncation below
    step^2 / 6 of a third derivative (at most 1/4 per unit of |dl|, 3 of |dh|
    here), rounding the results' bounds over the step."""
    rng = np.random.default_rng(96)
    z, idx = draw(rng, (5, 40), F32), rng.integers(0, 40, (5, 2))
    dl, dh, step = draw(rng, (5, 2), F32), draw(rng, 5, F32), F32(2.0 ** -4)

    def loss(z):
        r = run(z, idx, 1.0, 0, False, want=("logp", "entropy"))
        return (r["logp"].astype(np.float64) * dl).sum(1) + r["entropy"].astype(np.float64) * dh
    g = compare_grad(z, idx, 1.0, dl, dh, 1.0, F32)
    r = ot.logprobs(z.astype(np.float64), idx, 1.0, 0)
    noise = (r["logp_err"] * abs(dl)).sum(1) + r["entropy_err"] * abs(dh) + 10 * 2.0 ** -24 * (abs(dl).sum(1) + abs(dh))
    for j in range(40):
        up, down = z.copy(), z.copy()
        up[:, j] += step
        down[:, j] -= step
        d = (loss(up) - loss(down)) / (up[:, j].astype(np.float64) - down[:, j])
        lim = step ** 2 / 6 * (abs(dl).sum(1) / 4 + 3 * abs(dh)) + 2 * noise / step
        assert (abs(d - g[:, j]) <= lim).all(), j


def test_many_rows_gradient():
    rng = np.random.default_rng(97)
    z, idx = draw(rng, (1500, 300), F16), given(rng, 1500, 300, 1)
    compare_grad(z, idx, 1.0, draw(rng, (1500, 1), F32), None, 1.0, F8)


def test_captured_calls():
    rng = np.random.default_rng(98)
    for N, V in ((40, 3000), (2, 60000)):
        z, idx = dev(draw(rng, (N, V), F16)), dev(given(rng, N, V, 2))
        out = dict(logp=torch.empty((N, 2), device=DEV), entropy=torch.empty(N, device=DEV),
                   stats=torch.empty((N, 2), device=DEV),
                   top_idx=torch.empty((N, 9), dtype=torch.int64, device=DEV),
                   top_logp=torch.empty((N, 9), device=DEV))
        g, dl = torch.empty((N, V), dtype=torch.uint8, device=DEV), dev(draw(rng, (N, 2), F32))
        n = fp8t.token_logprobs_workspace_size(z, 9)
        ws = workspace(n)

        def call():
            fp8t.token_logprobs(z, idx, 1.0, **out, workspace=ws, workspace_bytes=n)
            fp8t.token_logprobs_bwd(z, idx, 1.0, out["stats"], out["entropy"], dl, out["entropy"], 8.0, g)
        replayed(call, [*out.values(), g])
