"""distill_loss against the float64 definition (oracle/lm.py) within the bounds
that it derives, and its gradient against difference quotients of its loss."""
import numpy as np
import pytest
import torch

import oracle
import paper_1812_08011_amd as fp8t
from oracle import lm
from tests.gpu_util import DEV, dev, host, say
from tests.lm_util import check, codes16, value

pytestmark = pytest.mark.gpu

TORCH = {np.float32: torch.float32, np.uint16: torch.uint16, np.uint8: torch.uint8}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    fp8t.lib()
    yield


def inputs(seed, N, V, k, z_type=np.float32, t_type=np.float32, std=2.0):
    rng = np.random.default_rng(seed)
    make = lambda shape, ty: (rng.standard_normal(shape) * std).astype(np.float32) \
        if ty == np.float32 else codes16(rng, shape, std)
    z, t = make((N, V), z_type), make((N, k), t_type)
    idx = np.stack([rng.choice(V, min(k, V), replace=False) for _ in range(N)]) if k <= V else \
        rng.integers(0, V, (N, k))
    return z, idx.astype(np.int64).reshape(N, k), t, rng.uniform(0.5, 2.0, N).astype(np.float32)


def run(z, idx, t, w, tau, scale, g_type, pad=0, shift=0, want=("loss", "g")):
    N, V = z.shape
    wide = np.full((N, V + pad + shift), 3, z.dtype)
    wide[:, shift:shift + V] = z
    zd = dev(wide)[:, shift:shift + V]
    gw = torch.full((N, V + pad + shift), 0x5A, dtype=torch.int32, device=DEV).to(TORCH[g_type])
    loss = torch.full((N,), np.nan, dtype=torch.float32, device=DEV)
    fp8t.distill_loss(zd, dev(idx), dev(t), None if w is None else dev(w), tau, scale,
                      loss if "loss" in want else None,
                      gw[:, shift:shift + V] if "g" in want else None)
    gh = host(gw).copy()
    g = gh[:, shift:shift + V].copy()
    gh[:, shift:shift + V] = 0x5A
    assert (gh == 0x5A).all(), "written outside the rows"
    return host(loss), g


def compare(z, idx, t, w, tau, scale, g_type, **kw):
    say(f"distill {z.shape} k={idx.shape[1]} {z.dtype} -> {g_type.__name__} tau={tau} {kw}")
    loss, g = run(z, idx, t, w, tau, scale, g_type, **kw)
    f32 = lambda x: np.float64(np.float32(x))
    want = lm.distill(value(z), idx, value(t), np.ones(len(z)) if w is None else w.astype(np.float64),
                      f32(tau), f32(scale))
    check("loss", loss, want[0], want[2])
    check("g", g, want[1], want[3])


@pytest.mark.parametrize("g_type", [np.float32, np.uint16, np.uint8])
@pytest.mark.parametrize("t_type", [np.float32, np.uint16])
@pytest.mark.parametrize("z_type", [np.float32, np.uint16])
def test_formats(z_type, t_type, g_type):
    compare(*inputs(30, 9, 777, 12, z_type, t_type), 2.0, 1024.0, g_type)


@pytest.mark.parametrize("V", [1, 2, 7, 63, 64, 65, 511, 4096, 6000, 8191, 20001, 70000, 131072,
                               150001, 300007])
@pytest.mark.parametrize("z_type", [np.float32, np.uint16])
def test_widths(V, z_type):
    compare(*inputs(31, 3, V, min(V, 10), z_type), 1.0, 512.0,
            np.uint16 if z_type == np.uint16 else np.float32)


@pytest.mark.parametrize("k", [1, 2, 64, 65, 300, 1000, 4096])
def test_top_counts(k):
    compare(*inputs(32, 4, 5000, k, np.uint16), 4.0, 64.0, np.uint16)


@pytest.mark.parametrize("pad,shift", [(0, 1), (5, 0), (8, 8), (3, 2)])
@pytest.mark.parametrize("z_type", [np.float32, np.uint16])
def test_row_strides_and_addresses(pad, shift, z_type):
    for V in (100, 2048, 9001):
        compare(*inputs(33, 5, V, 6, z_type), 2.0, 16.0, np.uint8, pad=pad, shift=shift)


def test_rows_without_a_target():
    """Weight 0, no used entry, every teacher logit -Inf: +0 whatever the
    logits hold; unused entries' logits are not looked at."""
    z, idx, t, w = inputs(34, 6, 500, 5)
    w[0] = 0.0
    z[0, 7] = np.nan
    idx[1] = -1
    t[1] = np.nan
    z[1, 3] = np.inf
    t[2] = -np.inf
    idx[3, 1:4] = [-1, 500, 2 ** 40]
    t[3, 1:4] = [np.nan, np.inf, 3e38]
    t[4, 2] = -np.inf
    for g_type in (np.float32, np.uint16, np.uint8):
        loss, g = run(z, idx, t, w, 1.5, 10.0, g_type)
        assert (loss[:3] == 0).all() and not np.signbit(loss[:3]).any()
        assert (g[:3] == 0).all() and not np.signbit(value(g[:3])).any()
        want = lm.distill(z[3:].astype(np.float64), idx[3:], t[3:].astype(np.float64),
                          w[3:].astype(np.float64), 1.5, 10.0)
        check("loss", loss[3:], want[0], want[2])
        check("g", g[3:], want[1], want[3])


def test_repeated_entries_and_masked_logits():
    z, idx, t, w = inputs(35, 4, 300, 6)
    idx[0] = 17                                       # one entry six times
    idx[1, :4] = [5, 9, 5, 9]
    z[2, 100:] = -np.inf                              # masked vocabulary
    idx[2] = [1, 2, 3, 4, 5, 6]
    z[3, :] = -3e38                                   # the type's lowest values, one at the teacher's
    z[3, idx[3, 0]] = 1.0
    t[3, 1:] = -np.inf
    compare(z, idx, t, w, 2.0, 1.0, np.float32)
    # the teacher on a masked entry: infinite loss, a finite gradient
    z, idx, t, w = inputs(36, 2, 300, 3)
    z[0, idx[0, 0]] = -np.inf
    loss, g = run(z, idx, t, w, 2.0, 1.0, np.float32)
    assert np.isposinf(loss[0]) and np.isfinite(g).all() and np.isfinite(loss[1])


def test_rows_that_are_not_finite_stay_alone():
    z, idx, t, w = inputs(37, 5, 1000, 4)
    clean = run(z, idx, t, w, 1.0, 1.0, np.float32)
    z2 = z.copy()
    z2[1, 5], z2[3, 7] = np.nan, np.inf
    loss, g = run(z2, idx, t, w, 1.0, 1.0, np.float32)
    assert np.isnan(loss[1]) and not np.isfinite(loss[3])
    assert np.isnan(g[1]).all() and np.isnan(g[3]).any()
    keep = [0, 2, 4]
    assert np.array_equal(loss[keep], clean[0][keep]) and np.array_equal(g[keep], clean[1][keep])


def test_large_logits_and_weights():
    z, idx, t, w = inputs(38, 4, 2000, 8, np.uint16, std=300.0)
    compare(z, idx, t, w, 1.0, 65536.0, np.uint16)
    z, idx, t, w = inputs(39, 4, 2000, 8)
    compare(z, idx, t, None, 3.0, -2.0, np.float32)


def test_one_of_two_results_and_in_place():
    say("distill, optional results and in place")
    for z_type, V in ((np.uint16, 6000), (np.float32, 501), (np.uint16, 140003), (np.float32, 140003)):
        z, idx, t, w = inputs(40, 4, V, 9, z_type)
        loss, g = run(z, idx, t, w, 2.0, 256.0, z_type)
        assert np.array_equal(run(z, idx, t, w, 2.0, 256.0, z_type, want=("loss",))[0], loss)
        assert np.array_equal(run(z, idx, t, w, 2.0, 256.0, z_type, want=("g",))[1], g)
        zd = dev(z)
        fp8t.distill_loss(zd, dev(idx), dev(t), dev(w), 2.0, 256.0, None, zd)
        assert np.array_equal(host(zd), g)


def test_gradient_is_the_difference_quotient():
    """Central differences of the FP32 loss: steps of 2^-4, whose truncation
    error is below h^2 / 6 of a third derivative (at most 1/4 tau^-1 w) and
    whose rounding error is the loss's over the step."""
    z, idx, t, w = inputs(41, 6, 40, 5)
    tau, h = 2.0, 2.0 ** -4
    f = lambda z: run(z, idx, t, w, tau, 1.0, np.float32)
    _, g = f(z)
    err = lm.distill(z.astype(np.float64), idx, t.astype(np.float64), w.astype(np.float64), tau, 1.0)[2]
    rng = np.random.default_rng(42)
    for _ in range(30):
        n, j = rng.integers(0, 6), rng.integers(0, 40)
        up, down = z.copy(), z.copy()
        up[n, j] += h
        down[n, j] -= h
        dz = float(up[n, j]) - float(down[n, j])
        d = (float(f(up)[0][n]) - float(f(down)[0][n])) / dz
        assert abs(d - g[n, j]) <= h * h / 6 * w[n] * tau + 2 * err[n] / h + 1e-6, (n, j)


def test_many_rows():
    z, idx, t, w = inputs(43, 1500, 300, 7, np.uint16)
    compare(z, idx, t, w, 2.0, 1024.0, np.uint8)
    empty = np.zeros((0, 5), np.float32)
    run(empty, np.zeros((0, 2), np.int64), np.zeros((0, 2), np.float32), np.zeros(0, np.float32), 1.0,
        1.0, np.float32)
