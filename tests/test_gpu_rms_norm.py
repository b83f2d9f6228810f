"""rms_norm_fwd and rms_norm_bwd against the float64 definitions
(oracle/tokens.py) within the bounds that they derive; the sum h bit for bit."""
import numpy as np
import pytest
import torch

import paper_1812_08011_amd as fp8t
from oracle import tokens as ot
from tests.gpu_util import DEV, dev, host, say
from tests.lm_util import check, value
from tests.token_util import F8, F16, F32, TORCH, Wide, draw, gpu, replayed, rounded, workspace  # noqa: F401

pytestmark = pytest.mark.gpu
WIDTHS = [1, 7, 8, 9, 64, 65, 128, 129, 200, 256, 257, 511, 512, 513, 1000, 1024, 1025, 2048, 2049, 4096, 4099, 8192, 8200, 16384,
          16385, 40003]


def fwd(x, r, w, eps, y_ty, s_ty=None, y_scale=1.0, rows=False, div=None, pad=0, shift=0, keep_h=True):
    """Checks a call and returns its results."""
    T, W = x.shape
    s_ty = s_ty or (F32 if r is None else r.dtype.type)
    say(f"rms_norm_fwd {T}x{W} x={x.dtype} r={None if r is None else r.dtype} h={keep_h and s_ty.__name__} "
        f"y={y_ty.__name__} rows={rows} {pad} {shift}")
    f32 = lambda v: value(v).astype(F32)
    u = f32(x)
    if div is not None:
        u = u / div[:, None]
    if r is not None:
        u = u + f32(r)
    if r is not None or keep_h:
        codes = rounded(u, s_ty)
        u = f32(codes)
    put = lambda a: None if a is None else Wide(T, W, a.dtype.type, pad, shift, a).view
    h = Wide(T, W, s_ty, pad, shift) if keep_h else None
    y = Wide(T, W, y_ty, pad, shift)
    scales = torch.full((T,), np.nan, device=DEV) if rows else None
    rstd = torch.full((T,), np.nan, device=DEV)
    fp8t.rms_norm_fwd(put(x), put(r), None if w is None else dev(w), eps, h.view if keep_h else None, y.view,
                      y_scale, scales, rstd, None if div is None else dev(div))
    got = dict(y=y.result(), rstd=host(rstd), h=h.result() if keep_h else None,
               scales=host(scales) if rows else None)
    if keep_h:
        same = (got["h"] == codes) | (np.isnan(value(codes)) & np.isnan(value(got["h"])))
        assert same.all(), np.argwhere(~same)[:5]
    want = ot.norm(u.astype(np.float64), np.ones(W) if w is None else value(w), float(np.float32(eps)),
                   float(np.float32(y_scale)), rows)
    for n in ("rstd", "y") + (("scales",) if rows else ()):
        check(n, got[n], want[n], want[n + "_err"])
    return got


@pytest.mark.parametrize("y", [F32, F16, F8])
@pytest.mark.parametrize("w", [None, F32, F16])
@pytest.mark.parametrize("s", [None, F32, F16])
@pytest.mark.parametrize("x", [F32, F16])
def test_forward_formats(x, s, w, y):
    rng = np.random.default_rng(60)
    T, W = 7, 300
    args = (draw(rng, (T, W), x), None if s is None else draw(rng, (T, W), s, 3.0),
            None if w is None else draw(rng, W, w), 1e-5, y)
    for rows in (False, True):
        fwd(*args, rows=rows, y_scale=28672.0 if rows else 1.5)
        fwd(*args, rows=rows, y_scale=3.0, s_ty=F16 if s is None else None)
        fwd(*args, rows=rows, y_scale=3.0, keep_h=False)


@pytest.mark.parametrize("W", WIDTHS)
def test_forward_widths_and_addresses(W):
    rng = np.random.default_rng(61)
    for T in (1, 5):
        x, r, w = draw(rng, (T, W), F16), draw(rng, (T, W), F32, 2.0), draw(rng, W, F16)
        fwd(x, r, w, 1e-6, F8, rows=True, y_scale=448.0)
        fwd(x, r, w, 1e-6, F8, pad=2, shift=1)
        fwd(x, None, None, 1e-6, F16, keep_h=False, pad=1, shift=1)
        fwd(x, draw(rng, (T, W), F16), w, 1e-6, F32, rows=True, y_scale=1.0, pad=3, shift=2)


def test_forward_in_place():
    """h in r's and in x's place."""
    rng = np.random.default_rng(62)
    for W in (100, 3001, 20000):
        say(f"rms_norm_fwd in place, {W}")
        x, r, w = draw(rng, (3, W), F16), draw(rng, (3, W), F16), draw(rng, W, F16)
        want = fwd(x, r, w, 1e-5, F8, rows=True, y_scale=100.0)
        for place in (0, 1):
            xd, rd, y = dev(x), dev(r), torch.empty((3, W), dtype=torch.uint8, device=DEV)
            scales = torch.empty(3, device=DEV)
            fp8t.rms_norm_fwd(xd, rd, dev(w), 1e-5, rd if place else xd, y, 100.0, scales)
            assert np.array_equal(host(rd if place else xd), want["h"])
            assert np.array_equal(host(y), want["y"]) and np.array_equal(host(scales), want["scales"])


def test_forward_one_result_at_a_time():
    rng = np.random.default_rng(63)
    x, r, w = draw(rng, (4, 700), F16), draw(rng, (4, 700), F32), draw(rng, 700, F16)
    want = fwd(x, r, w, 1e-5, F16)
    h, y, rstd = torch.empty((4, 700), device=DEV), dev(x), torch.empty(4, device=DEV)
    fp8t.rms_norm_fwd(dev(x), dev(r), dev(w), 1e-5, h, None)
    fp8t.rms_norm_fwd(dev(x), dev(r), dev(w), 1e-5, None, None, rstd=rstd)
    fp8t.rms_norm_fwd(dev(x), dev(r), dev(w), 1e-5, None, y)
    assert np.array_equal(host(h), want["h"]) and np.array_equal(host(rstd), want["rstd"])
    assert np.array_equal(host(y), want["y"])


def test_forward_far_magnitudes():
    """Squares past FP32's range, rows of zeros, rows below eps."""
    rng = np.random.default_rng(64)
    for W in (50, 3000, 20000):
        x = draw(rng, (6, W), F32)
        x[0] *= F32(1e30)
        x[1] *= F32(1e-30)
        x[2] = 0
        x[3] *= F32(2.0 ** 62)
        x[4] *= F32(3e-5)
        for rows in (False, True):
            got = fwd(x, None, None, 1e-9, F32, rows=rows, y_scale=2.0, keep_h=False)
        assert got["scales"][2] == 1.0 and (got["y"][2] == 0).all()
        fwd(x, None, None, 2.0 ** -100, F32, keep_h=False)
        codes = np.full((2, W), 0x7DFF, F16)                       # the largest FP16 value
        codes[1] = 1                                               # the smallest
        fwd(codes, None, None, 1e-5, F32, keep_h=False)


def test_forward_rows_that_are_not_finite_stay_alone():
    rng = np.random.default_rng(65)
    for W in (60, 1500, 20000):
        x, r = draw(rng, (9, W), F16), draw(rng, (9, W), F32)
        clean = fwd(x, r, None, 1e-5, F8, rows=True, y_scale=64.0)
        bad = r.copy()
        bad[1, 3], bad[4, W - 1], bad[6, 0] = np.nan, np.inf, -np.inf
        say("rms_norm_fwd rows that are not finite")
        y, scales = torch.empty((9, W), dtype=torch.uint8, device=DEV), torch.empty(9, device=DEV)
        rstd = torch.empty(9, device=DEV)
        fp8t.rms_norm_fwd(dev(x), dev(bad), None, 1e-5, None, y, 64.0, scales, rstd)
        keep = [0, 2, 3, 5, 7, 8]
        assert np.array_equal(host(y)[keep], clean["y"][keep])
        assert np.array_equal(host(scales)[keep], clean["scales"][keep])
        got = value(host(y))
        assert np.isnan(got[1]).all() and np.isnan(got[4, W - 1]) and np.isnan(got[6, 0])
        assert (host(scales)[[1, 4, 6]] == 1.0).all()
        assert np.isnan(host(rstd)[1]) and (host(rstd)[[4, 6]] == 0).all()


def test_scaled_rows_are_divided_again():
    """y with each row's own scale, and a product of it, given to the next norm:
    as if there had been no scale."""
    rng = np.random.default_rng(66)
    x, r = draw(rng, (20, 96), F16), draw(rng, (20, 96), F32)
    got = fwd(x, r, None, 1e-5, F16, rows=True, y_scale=2.0 ** 20)
    fwd(got["y"], got["h"], None, 1e-5, F8, div=got["scales"])
    fwd(draw(rng, (20, 20000), F16), None, None, 1e-5, F8, div=got["scales"])


def bwd(h, w, rstd, dy, dr, d_ty, dw_ty=F32, s8=1.0, pad=0, shift=0, want_of=("dx", "dx8", "dw")):
    T, W = h.shape
    say(f"rms_norm_bwd {T}x{W} h={h.dtype} dy={dy.dtype} d={d_ty.__name__} dr={dr is not None} "
        f"dw={dw_ty.__name__} {pad} {shift}")
    put = lambda a: None if a is None else Wide(T, W, a.dtype.type, pad, shift, a).view
    dx, dx8 = Wide(T, W, d_ty, pad, shift), Wide(T, W, F8, pad, shift)
    dw = torch.full((W,), 7, dtype=torch.int32, device=DEV).to(TORCH[dw_ty])
    hd = put(h)
    n = fp8t.rms_norm_bwd_workspace_size(hd) if "dw" in want_of else 0
    fp8t.rms_norm_bwd(hd, None if w is None else dev(w), dev(rstd), put(dy), put(dr),
                      dx.view if "dx" in want_of else None, dx8.view if "dx8" in want_of else None, s8,
                      dw if "dw" in want_of else None, workspace(n), n)
    got = dict(dx=dx.result(), dx8=dx8.result(), dw=host(dw))
    d, err, dwv, dw_err = ot.norm_grad(value(h), np.ones(W) if w is None else value(w),
                                       rstd.astype(np.float64), value(dy), None if dr is None else value(dr))
    s8 = float(np.float32(s8))
    if "dx" in want_of:
        check("dx", got["dx"], d, err)
    if "dx8" in want_of:
        check("dx8", got["dx8"], d * s8, abs(s8) * (err + abs(d) * 2.0 ** -23))
    if "dw" in want_of:
        check("dw", got["dw"], dwv, dw_err)
    return got


def inverse_rms(h, eps=1e-5):
    return (1.0 / np.sqrt((value(h) ** 2).mean(1) + eps)).astype(F32)


@pytest.mark.parametrize("d", [F32, F16])
@pytest.mark.parametrize("dy", [F32, F16, F8])
@pytest.mark.parametrize("w", [None, F32, F16])
@pytest.mark.parametrize("h", [F32, F16])
def test_gradient_formats(h, w, dy, d):
    rng = np.random.default_rng(67)
    T, W = 11, 300
    hv = draw(rng, (T, W), h, 2.0)
    for dr in (None, draw(rng, (T, W), d)):
        bwd(hv, None if w is None else draw(rng, W, w), inverse_rms(hv), draw(rng, (T, W), dy), dr, d,
            F16 if d == F16 else F32, 3.0)


@pytest.mark.parametrize("W", WIDTHS)
def test_gradient_widths_and_addresses(W):
    rng = np.random.default_rng(68)
    for T in (1, 2, 9):
        h, w = draw(rng, (T, W), F16), draw(rng, W, F16)
        dy, dr = draw(rng, (T, W), F16), draw(rng, (T, W), F32)
        bwd(h, w, inverse_rms(h), dy, dr, F32)
        bwd(h, w, inverse_rms(h), dy, None, F16, pad=2, shift=1)


@pytest.mark.parametrize("T,W", [(0, 40), (3, 40), (1023, 40), (5000, 9), (3001, 100), (3001, 250), (5003, 600), (1500, 2100),
                                 (700, 5000), (300, 9000), (200, 17000)])
def test_gradient_many_rows(T, W):
    rng = np.random.default_rng(69)
    h, w = draw(rng, (T, W), F16), draw(rng, W, F32)
    bwd(h, w, inverse_rms(h) if T else np.zeros(0, F32), draw(rng, (T, W), F8), draw(rng, (T, W), F16), F16)


def test_gradient_one_result_at_a_time_and_in_place():
    rng = np.random.default_rng(70)
    for W in (200, 3000, 17000):
        h, w = draw(rng, (5, W), F32), draw(rng, W, F16)
        args = (h, w, inverse_rms(h), draw(rng, (5, W), F16), draw(rng, (5, W), F32), F32)
        want = bwd(*args)
        for n in ("dx", "dx8", "dw"):
            assert np.array_equal(bwd(*args, want_of=(n,))[n], want[n])
        dr = dev(args[4])
        fp8t.rms_norm_bwd(dev(h), dev(w), dev(args[2]), dev(args[3]), dr, dr)
        assert np.array_equal(host(dr), want["dx"])


def test_gradient_is_the_difference_quotient():
    """Central differences of <y, e> in FP32, step 2^-5: the truncation is below
    step^2 / 6 of a third derivative (the norm's are below 15 rstd^3 |e| here),
    the rounding that of 40 FP32 results over the step."""
    rng = np.random.default_rng(71)
    h, w, e = draw(rng, (3, 40), F32), draw(rng, 40, F32), draw(rng, (3, 40), F32)

    def loss(h, w):
        y = torch.empty((3, 40), device=DEV)
        fp8t.rms_norm_fwd(dev(h), None, dev(w), 1e-5, None, y)
        return (host(y).astype(np.float64) * e).sum(1)
    got = bwd(h, w, inverse_rms(h), e, None, F32)
    step = F32(2.0 ** -5)
    mag = abs(e).sum(1) * abs(w).max() * inverse_rms(h)
    for j in range(40):
        up, down = h.copy(), h.copy()
        up[:, j] += step
        down[:, j] -= step
        diff = (up[:, j].astype(np.float64) - down[:, j])
        d = (loss(up, w) - loss(down, w)) / diff
        lim = step ** 2 / 6 * 15 * inverse_rms(h) ** 2 * mag + 2 * mag * 40 * 2.0 ** -23 / step
        assert (abs(d - got["dx"][:, j]) <= lim).all(), j
        up, down = w.copy(), w.copy()
        up[j] += step
        down[j] -= step
        d = ((loss(h, up) - loss(h, down)) / (up[j].astype(np.float64) - down[j])).sum()
        assert abs(d - got["dw"][j]) <= 2 * mag.sum() * 40 * 2.0 ** -23 / step, j


def test_gradient_rows_that_are_not_finite_stay_alone():
    rng = np.random.default_rng(72)
    for W in (60, 1500, 17000):
        h, w, dy = draw(rng, (6, W), F16), draw(rng, W, F16), draw(rng, (6, W), F16)
        rstd = inverse_rms(h)
        clean = bwd(h, w, rstd, dy, None, F32)
        bad = dy.copy()
        bad[2, 5] = 0x7F00                                        # NaN
        say("rms_norm_bwd rows that are not finite")
        dx = torch.empty((6, W), device=DEV)
        fp8t.rms_norm_bwd(dev(h), dev(w), dev(rstd), dev(bad), None, dx)
        got = host(dx)
        assert np.isnan(got[2]).all() and np.array_equal(np.delete(got, 2, 0), np.delete(clean["dx"], 2, 0))


def test_captured_calls():
    rng = np.random.default_rng(73)
    x, r, w = dev(draw(rng, (300, 600), F16)), dev(draw(rng, (300, 600), F32)), dev(draw(rng, 600, F16))
    h, y = torch.empty((300, 600), device=DEV), torch.empty((300, 600), dtype=torch.uint8, device=DEV)
    rstd, scales = torch.empty(300, device=DEV), torch.empty(300, device=DEV)
    dx, dw = torch.empty((300, 600), device=DEV), torch.empty(600, device=DEV)
    n = fp8t.rms_norm_bwd_workspace_size(h)
    ws = workspace(n)

    def call():
        fp8t.rms_norm_fwd(x, r, w, 1e-5, h, y, 64.0, scales, rstd)
        fp8t.rms_norm_bwd(h, w, rstd, y, r, dx, None, 1.0, dw, ws, n)
    replayed(call, [h, y, rstd, scales, dx, dw])
