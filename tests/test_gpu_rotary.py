"""rotary_embed and fp16_dequantize against their definitions."""
import numpy as np
import pytest
import torch

import oracle
import paper_1812_08011_amd as fp8t
from oracle import lm
from tests.gpu_util import DEV, dev, host, say
from tests.lm_util import P16, check, codes16, codes8, value

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    fp8t.lib()
    yield


@pytest.mark.parametrize("shift", [0, 1])
def test_dequantize_every_code(shift):
    say("fp16_dequantize, every code, shift", shift)
    codes = np.arange(65536, dtype=np.uint16)[shift:]
    src = dev(np.arange(65536, dtype=np.uint16))[shift:]
    f = torch.empty(codes.size + shift, dtype=torch.float32, device=DEV)[shift:]
    fp8t.fp16_dequantize(src, f)
    want = P16[codes].astype(np.float32)
    assert np.array_equal(host(f), want, equal_nan=True)
    h = torch.empty(codes.size + shift, dtype=torch.float16, device=DEV)[shift:]
    for scale in (1.0, 0.37):
        fp8t.fp16_dequantize(src, h, scale)
        with np.errstate(over="ignore"):
            assert np.array_equal(host(h), (want * np.float32(scale)).astype(np.float16), equal_nan=True)


TYPES = {"f32": (np.float32, torch.float32), "fp16": (np.uint16, torch.uint16),
         "fp8": (np.uint8, torch.uint8)}


def make(rng, kind, shape):
    if kind == "f32":
        return rng.standard_normal(shape).astype(np.float32)
    return codes16(rng, shape) if kind == "fp16" else codes8(rng, shape)


def turned(x, pos, freqs, y_kind, interleaved, inverse, mscale, scale, want_x):
    y = torch.empty(x.shape, dtype=TYPES[y_kind][1], device=DEV)
    fp8t.rotary_embed(x, dev(pos), dev(freqs), y, interleaved, inverse, mscale, scale)
    ref = lm.rotary(want_x, pos, freqs, interleaved, inverse, mscale) * scale
    # cos and sin: the angle's fraction of a turn in FP32 (2 pi 2^-26), the
    # functions 4 steps of 2^-24; two products and their sum, the scale: 8 EPS32
    R = 2 * len(freqs)
    err = np.zeros_like(want_x)
    n = len(freqs)
    i0 = 2 * np.arange(n) if interleaved else np.arange(n)
    i1 = i0 + 1 if interleaved else i0 + n
    pair = abs(want_x[..., i0]) + abs(want_x[..., i1])
    err[..., i0] = err[..., i1] = pair * abs(mscale * scale) * (2 * np.pi * 2.0 ** -26 + 12 * 2.0 ** -24)
    err[..., R:] = abs(want_x[..., R:] * scale) * 2.0 ** -24
    check("y", host(y), ref, err)
    return y


@pytest.mark.parametrize("y_kind", ["f32", "fp16", "fp8"])
@pytest.mark.parametrize("x_kind", ["f32", "fp16", "fp8"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_formats(x_kind, y_kind, interleaved):
    say(f"rotary {x_kind} -> {y_kind} interleaved={interleaved}")
    rng = np.random.default_rng(20)
    x = make(rng, x_kind, (37, 3, 64))
    pos = rng.integers(0, 4000, 37)
    freqs = 10000.0 ** -(np.arange(32) / 32)
    for inverse in (False, True):
        turned(dev(x), pos, freqs, y_kind, interleaved, inverse, 1.25, 1.0, value(x))


@pytest.mark.parametrize("D,R", [(128, 128), (128, 32), (80, 48), (100, 100), (7, 4), (2, 2), (5, 0),
                                 (1, 0), (33, 32), (512, 512), (64, 8)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_sizes_and_parts(D, R, interleaved):
    say(f"rotary D={D} R={R} interleaved={interleaved}")
    rng = np.random.default_rng(21)
    for T, H in ((1, 1), (3, 5), (70, 2)):
        x = make(rng, "fp16", (T, H, D))
        pos = rng.integers(-50, 100000, T)
        freqs = 500000.0 ** -(np.arange(R // 2) / max(1, R // 2))
        turned(dev(x), pos, freqs, "fp8", interleaved, False, 1.0, 4.0, value(x))
        turned(dev(x), pos, freqs, "fp16", interleaved, True, 0.7, 1.0, value(x))


@pytest.mark.parametrize("interleaved", [False, True])
def test_far_positions_keep_their_accuracy(interleaved):
    say("rotary, far positions")
    rng = np.random.default_rng(22)
    pos = np.array([2 ** 20 + 1, 2 ** 31 - 1, 2 ** 31 + 5, -(2 ** 33), 0, 1])
    x = make(rng, "f32", (6, 2, 16))
    # beyond 2^33 radians the product position x freq / (2 pi) itself is off by
    # 2^-53 of 2^31 turns or less: below FP32's fraction
    turned(dev(x), pos, 10.0 ** -np.arange(8.0), "f32", interleaved, False, 1.0, 1.0, value(x))


@pytest.mark.parametrize("kind", ["f32", "fp16", "fp8"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,R,off", [(64, 64, 0), (64, 64, 3), (72, 40, 1), (128, 64, 0)])
def test_strides_and_in_place(kind, interleaved, D, R, off):
    """Heads inside a wider projection, turned in place, the rest untouched."""
    say(f"rotary in place {kind} D={D} R={R} off={off}")
    rng = np.random.default_rng(23)
    wide = make(rng, kind, (19, 6, D + 2 * off))
    pos, freqs = np.arange(19) * 7, 10000.0 ** -(np.arange(R // 2) / (R // 2))
    buf = dev(wide)
    part = buf[:, 1:4, off:off + D]
    alone = turned(part, pos, freqs, kind, interleaved, False, 1.0, 1.0,
                   value(wide[:, 1:4, off:off + D]))
    fp8t.rotary_embed(part, dev(pos), dev(freqs), part, interleaved)
    got = host(buf)
    assert np.array_equal(got[:, 1:4, off:off + D], host(alone))
    got = got.copy()
    got[:, 1:4, off:off + D] = wide[:, 1:4, off:off + D]
    assert np.array_equal(got, wide)


def test_values_that_are_not_finite_stay_in_their_pair():
    say("rotary, NaN and Inf")
    rng = np.random.default_rng(24)
    x = make(rng, "fp16", (4, 2, 32))
    x[1, 0, 3], x[2, 1, 30] = 0x7F00, 0x7E00
    pos, freqs = np.arange(1, 5), 100.0 ** -(np.arange(8) / 8)
    y = torch.empty((4, 2, 32), dtype=torch.uint8, device=DEV)
    fp8t.rotary_embed(dev(x), dev(pos), dev(freqs), y)
    bad = np.argwhere(~np.isfinite(value(host(y))))
    assert sorted(map(tuple, bad)) == [(1, 0, 3), (1, 0, 11), (2, 1, 30)]


def test_large_rows_and_many_tokens():
    say("rotary, many tokens")
    rng = np.random.default_rng(25)
    x = make(rng, "fp16", (3001, 9, 128))
    pos, freqs = rng.integers(0, 1 << 17, 3001), 10000.0 ** -(np.arange(64) / 64)
    turned(dev(x), pos, freqs, "fp8", False, False, 1.0, 1.0, value(x))
    turned(dev(x), pos, freqs, "fp8", True, True, 1.0, 1.0, value(x))
