"""rms_norm_fwd bit for bit: what it rounds is stated, so that from the stored sum,
rstd and a row's scale every result follows in float32 products."""
import numpy as np
import pytest
import torch

import paper_1812_08011_amd as fp8t
from tests.gpu_util import DEV, dev, host, say
from tests.lm_util import value
from tests.token_util import F8, F16, F32, TORCH, draw, gpu, rounded  # noqa: F401

pytestmark = pytest.mark.gpu
WIDTHS = [1, 9, 64, 100, 200, 500, 1000, 2048, 4099, 8200, 16384, 20003]


def run(x, r, w, y_ty, rows, y_scale=1.0, eps=1e-5):
    """h, y, rstd and the rows' scales (None without)."""
    T, W = x.shape
    h = torch.empty((T, W), dtype=TORCH[x.dtype.type if r is None else r.dtype.type], device=DEV)
    y, rstd = torch.empty((T, W), dtype=TORCH[y_ty], device=DEV), torch.empty(T, device=DEV)
    scales = torch.empty(T, device=DEV) if rows else None
    put = lambda a: None if a is None else dev(a)
    say(f"rms_norm_fwd {T}x{W} {x.dtype} {None if r is None else r.dtype} -> {y_ty.__name__} rows={rows}")
    fp8t.rms_norm_fwd(dev(x), put(r), put(w), eps, h, y, y_scale, scales, rstd)
    return host(h), host(y), host(rstd), None if scales is None else host(scales)


def same(got, want):
    a, b = value(got), value(want)
    ok = (got == want) | (np.isnan(a) & np.isnan(b))
    assert ok.all(), [(tuple(i), a[tuple(i)], b[tuple(i)]) for i in np.argwhere(~ok)[:5]]


def products(h, rstd, w, y_scale, rows):
    """n, and its rows' scales, in float32."""
    with np.errstate(invalid="ignore", over="ignore", under="ignore", divide="ignore"):
        n = value(h).astype(F32) * rstd[:, None]
        if w is not None:
            n = n * value(w).astype(F32)
        c = np.full(len(n), F32(y_scale))
        if rows:
            top = abs(n).max(1)
            some = (top > 0) & np.isfinite(top)
            c = np.where(some, np.minimum(F32(y_scale) / np.where(some, top, F32(1)), F32(2.0 ** 126)), F32(1))
        return n * c[:, None], c


@pytest.mark.parametrize("rows", [False, True])
@pytest.mark.parametrize("W", WIDTHS)
def test_products_are_floats(W, rows):
    rng = np.random.default_rng(120)
    for x, r, w, y in ((F16, F32, F16, F8), (F32, None, F32, F16), (F16, F16, None, F32)):
        w = None if w is None else draw(rng, W, w)
        scale = 28672.0 if rows else 1.5
        h, got, rstd, c = run(draw(rng, (6, W), x), None if r is None else draw(rng, (6, W), r, 3.0), w, y, rows, scale)
        n, want = products(h, rstd, w, scale, rows)
        same(got, rounded(n, y))
        if rows:
            assert np.array_equal(c, want)


@pytest.mark.parametrize("ty", [F32, F16])
@pytest.mark.parametrize("W", [60, 1500, 9000, 20000])
def test_weights_that_are_not_finite(W, ty):
    """Inf and NaN among the weights follow IEEE arithmetic in their columns: an
    infinite weight times a value is Inf of its sign, times 0 is NaN."""
    rng = np.random.default_rng(121)
    inf, low, nan, big = (np.inf, -np.inf, np.nan, 3e38) if ty == F32 else (0x7E00, 0xFE00, 0x7F00, 0x7DFF)
    for x in (F32, F16):
        w, data = draw(rng, W, ty), draw(rng, (40, W), x)
        w[[1, W // 2, W - 1]], w[3], w[5], w[7] = inf, low, nan, big
        data[:, 1:4][rng.random((40, 3)) < 0.1] = 0
        for rows in (False, True):
            for y in (F32, F16, F8):
                h, got, rstd, c = run(data, None, w, y, rows, 2.0)
                n, want = products(h, rstd, w, 2.0, rows)
                assert np.isfinite(rstd).all() and np.isinf(n).any() and np.isnan(n).any()
                same(got, rounded(n, y))
                if rows:
                    assert (c == 1.0).all() and np.array_equal(c, want)


@pytest.mark.parametrize("W", WIDTHS + [300007])
def test_rstd_is_rounded_once(W):
    """Squares, their mean and 1 / rms are doubles: a sum of W terms is off by W
    2^-53 of itself, 2^-34 at the widest here, rstd by half of that and its last
    steps' 2^-50; then it is rounded to a float."""
    rng = np.random.default_rng(122)
    x = draw(rng, (5, W), F32)
    x[1] *= F32(1e30)                                          # squares past FP32's range
    x[2] *= F32(2.0 ** 62)
    x[3] = np.exp(rng.uniform(-60, 60, W)).astype(F32)
    x[4] *= F32(1e-30)
    for ty, data in ((F32, x), (F16, draw(rng, (40, W), F16, 2.0))):
        for eps in (1e-5, 2.0 ** -100):
            h, y, rstd, _ = run(data, None, None, F32, False, eps=eps)
            want = 1.0 / np.sqrt((value(h) ** 2).mean(1) + float(F32(eps)))
            assert (abs(rstd - want) <= want * (2.0 ** -24 + 2.0 ** -35 + 2.0 ** -50) + 2.0 ** -150).all(), \
                (abs(rstd / want - 1) * 2 ** 24).max()
