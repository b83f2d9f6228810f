"""embed_fwd bit for bit and embed_bwd against the float64 definition
(oracle/tokens.py) within the bound of its sums."""
import numpy as np
import pytest
import torch

import paper_1812_08011_amd as fp8t
from oracle import tokens as ot
from tests.gpu_util import DEV, dev, host, say
from tests.lm_util import check, value
from tests.token_util import F8, F16, F32, Wide, draw, gpu, replayed, rounded, workspace  # noqa: F401

pytestmark = pytest.mark.gpu


def fwd(tok, table, ty, scale, pad=0, shift=0):
    say(f"embed_fwd T={len(tok)} table={table.shape} {table.dtype} -> {ty.__name__} {pad} {shift}")
    V, W = table.shape
    t, y = Wide(V, W, table.dtype.type, pad, shift, table), Wide(len(tok), W, ty, pad, shift)
    fp8t.embed_fwd(dev(tok), t.view, y.view, scale)
    used = (tok >= 0) & (tok < V)
    want = np.zeros((len(tok), W), F32)
    want[used] = value(table[tok[used]]).astype(F32) * F32(scale)
    got, want = y.result(), rounded(want, ty)
    same = (got == want) | (np.isnan(value(got)) & np.isnan(value(want)))
    assert same.all(), np.argwhere(~same)[:5]


@pytest.mark.parametrize("ty", [F32, F16, F8])
@pytest.mark.parametrize("table", [F32, F16, F8])
def test_forward_formats(table, ty):
    rng = np.random.default_rng(50)
    tok = rng.integers(-2, 35, 77)
    fwd(tok, draw(rng, (33, 100), table), ty, 3.7)
    fwd(tok, draw(rng, (33, 96), table), ty, 0.0)


@pytest.mark.parametrize("W", [1, 7, 8, 9, 64, 513, 2048, 2051, 5000])
def test_forward_widths_and_addresses(W):
    rng = np.random.default_rng(51)
    for T in (0, 1, 2, 3, 33):
        fwd(rng.integers(0, 20, T), draw(rng, (20, W), F16), F8, 2.0, 3, 1)
        fwd(rng.integers(0, 20, T), draw(rng, (20, W), F32), F16, 2.0)


def test_forward_special_values_and_far_tokens():
    table = np.arange(65536, dtype=F16).reshape(256, 256)
    fwd(np.array([0, 255, 3, -1, 256, 2 ** 40, -2 ** 62, 252]), table, F32, 1.0)
    codes = np.arange(256, dtype=F8).reshape(2, 128)
    for ty in (F32, F16):
        say("embed_fwd every code")
        y = Wide(3, 128, ty)
        fp8t.embed_fwd(dev(np.array([1, 0, 1])), dev(codes), y.view, 1.0)
        got, want = value(y.result()), value(codes)[[1, 0, 1]]
        assert np.array_equal(got, want, equal_nan=True)


def bwd(tok, e, V, g_ty, scale, pad=0, shift=0):
    say(f"embed_bwd T={len(tok)} V={V} e={e.shape} {e.dtype} -> {g_ty.__name__} {pad} {shift}")
    T, W = e.shape
    ed, g = Wide(T, W, e.dtype.type, pad, shift, e), Wide(V, W, g_ty, pad, shift)
    td = dev(np.asarray(tok, np.int64))
    n = fp8t.embed_bwd_workspace_size(td, ed.view, g.view)
    fp8t.embed_bwd(td, ed.view, g.view, scale, workspace(n), n)
    got = g.result()
    want, err = ot.embed_grad(tok, value(e), V, float(np.float32(scale)))
    check("g", got, want, err + 2 * abs(want) * 2.0 ** -24)
    named = np.zeros(V, bool)
    named[tok[(tok >= 0) & (tok < V)]] = True
    assert not np.signbit(value(got[~named])).any() and (value(got[~named]) == 0).all()
    return got


@pytest.mark.parametrize("g", [F32, F16, F8])
@pytest.mark.parametrize("e", [F32, F16, F8])
def test_gradient_formats(e, g):
    rng = np.random.default_rng(52)
    bwd(rng.integers(-1, 60, 300), draw(rng, (300, 100), e), 57, g, 3.25)


@pytest.mark.parametrize("W", [3, 24, 260, 520, 1030])
@pytest.mark.parametrize("T", [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 129, 1000, 5000])
def test_gradient_run_lengths(T, W):
    """One token for all: runs that end before, at and behind the borders of
    the pieces, of their shares and of what is not cut; with other tokens, and
    long runs of theirs, before and behind."""
    rng = np.random.default_rng(53)
    e = draw(rng, (T, W), F16)
    bwd(np.full(T, 5), e, 9, F32, 1.0)
    for before in (1, 15, 16, 31, 33, 64, 200):
        tok = np.full(T + before + 140, 5)
        tok[:before], tok[T + before:] = 2, np.arange(140) % 3 + 6
        tok[T + before + 60:] = 8
        rng.shuffle(tok)
        bwd(tok, draw(rng, (len(tok), W), F16), 9, F32, 1.0)


@pytest.mark.parametrize("W", [1, 5, 8, 17, 64, 512, 513, 1024, 1500])
def test_gradient_widths_and_addresses(W):
    rng = np.random.default_rng(54)
    tok = rng.integers(0, 12, 400) ** 2 // 12
    bwd(tok, draw(rng, (400, W), F16), 13, F16, 2.0)
    bwd(tok, draw(rng, (400, W), F8), 13, F8, 2.0, 3, 1)


@pytest.mark.parametrize("V", [1, 2, 15, 16, 17, 255, 4096, 4097, 50001, 140000])
def test_gradient_vocabularies(V):
    rng = np.random.default_rng(55)
    tok = np.minimum((V ** rng.random(3000)).astype(np.int64), V) - 1
    tok[::50] = V - 1
    bwd(tok, draw(rng, (3000, 16), F16), V, F32, 1.0)


def test_gradient_tokens_in_any_order():
    rng = np.random.default_rng(56)
    V = 3000
    for tok in (np.arange(V), np.arange(V)[::-1].copy(), np.sort(rng.integers(0, V, 9000)),
                rng.integers(-50, V + 50, 20000), np.full(500, -1), np.full(500, V)):
        bwd(tok, draw(rng, (len(tok), 8), F16), V, F32, 1.0)


def test_gradient_of_many_tokens_is_summed_in_order():
    """More of its rows' tokens than a wave keeps: the second reading; the sum is
    that of the errors in the order of t, the same bits whatever lies between."""
    rng = np.random.default_rng(57)
    T = 30000
    tok = np.where(rng.random(T) < 0.8, rng.integers(0, 3, T), rng.integers(0, 900, T))
    e = draw(rng, (T, 8), F32)
    got = bwd(tok, e, 900, F32, 1.0)
    keep = np.argsort(tok, kind="stable")
    again = bwd(tok[keep], e[keep], 900, F32, 1.0)
    assert np.array_equal(got, again)


def test_gradient_far_values_stay_in_their_rows():
    rng = np.random.default_rng(58)
    tok = rng.integers(0, 10, 200)
    e = draw(rng, (200, 16), F32)
    clean = bwd(tok, e, 10, F32, 1.0)
    bad = e.copy()
    bad[7, 3], bad[8, 4] = np.nan, np.inf
    none = np.append(tok, [-1, 10])
    say("embed_bwd NaN and Inf, also in tokens of no row")
    td, ed = dev(none), dev(np.vstack([bad, np.full((2, 16), np.nan, F32)]))
    g = torch.empty((10, 16), device=DEV)
    n = fp8t.embed_bwd_workspace_size(td, ed, g)
    fp8t.embed_bwd(td, ed, g, 1.0, workspace(n), n)
    got = host(g)
    assert np.isnan(got[tok[7], 3]) and not np.isfinite(got[tok[8], 4])
    rest = np.ones((10, 16), bool)
    rest[tok[7], 3] = rest[tok[8], 4] = False
    assert np.array_equal(got[rest], clean[rest])


def test_gradient_is_the_adjoint():
    """<embed_fwd(table), e> = <table, embed_bwd(e)> in floats; each side is a
    sum of 60000 products, off by its results' roundings."""
    rng = np.random.default_rng(59)
    tok = rng.integers(-1, 40, 1000)
    table, e = draw(rng, (40, 60), F32), draw(rng, (1000, 60), F32)
    y, g = torch.empty((1000, 60), device=DEV), torch.empty((40, 60), device=DEV)
    td, ed = dev(tok), dev(e)
    fp8t.embed_fwd(td, dev(table), y, 1.5)
    n = fp8t.embed_bwd_workspace_size(td, ed, g)
    fp8t.embed_bwd(td, ed, g, 1.5, workspace(n), n)
    left = (host(y).astype(np.float64) * e).sum()
    right = (host(g).astype(np.float64) * table).sum()
    mag = abs(host(y).astype(np.float64) * e).sum()
    assert abs(left - right) <= mag * 2.0 ** -24 * (1000 / 40 * 3 + 8)


def test_captured_calls():
    rng = np.random.default_rng(60)
    td, ed = dev(np.minimum(rng.integers(0, 400, 2000), 200)), dev(draw(rng, (2000, 64), F16))
    table, y = dev(draw(rng, (300, 64), F16)), torch.empty((2000, 64), dtype=torch.uint8, device=DEV)
    g = torch.empty((300, 64), dtype=torch.uint16, device=DEV)
    n = fp8t.embed_bwd_workspace_size(td, ed, g)
    ws = workspace(n)

    def call():
        fp8t.embed_fwd(td, table, y, 2.0)
        fp8t.embed_bwd(td, ed, g, 2.0, ws, n)
    replayed(call, [y, g])
