"""attn_bwd_fp8 with errors and values of very different sizes in one call:
what a row's or a key's gradient keeps does not depend on other rows, other
sequences or tokens of no sequence."""
import numpy as np
import pytest
import torch

import oracle
import paper_1812_08011_amd as fp8t
from oracle import lm
from tests.gpu_util import say
from tests.lm_util import codes8, offsets, run_attention, value
from tests.test_gpu_attention import compare

pytestmark = pytest.mark.gpu
TOP8 = 0x7B                                            # 57344, the largest FP8 value


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    fp8t.lib()
    yield


def scaled(rng, shape, sizes):
    """Normal codes times one size a token."""
    x = rng.standard_normal(shape) * np.asarray(sizes, np.float64)[:, None, None]
    return oracle.fp8_quantize(x.astype(np.float32))


def run(seed, lens, Hq, Hkv, D, causal, e_sizes, v_sizes, grad_scale, top_e=(), top_v=()):
    rng = np.random.default_rng(seed)
    T, cu, c = sum(lens), offsets(lens), float(np.float32(1 / np.sqrt(D)))
    q, k = codes8(rng, (T, Hq, D)), codes8(rng, (T, Hkv, D))
    v, e = scaled(rng, (T, Hkv, D), v_sizes), scaled(rng, (T, Hq, D), e_sizes)
    for t in top_e:
        e[t] = TOP8
    for t in top_v:
        v[t] = TOP8
    got = run_attention(q, k, v, cu, cu, causal, c, e, np.uint16, (1.0, grad_scale))
    compare(got, lm.attention(value(q), value(k), value(v), cu, cu, causal, c, value(e)),
            (1.0, grad_scale))


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("bits", [10, 20, 26])
def test_sequences_of_different_errors(bits, D, causal):
    """One sequence's errors 2^-bits of the other's, one of whose rows is
    saturated; the loss scale brings the small gradients into FP16."""
    say(f"gradients, errors 2^-{bits} apart, D={D}, causal={causal}")
    lens = [200, 130]
    sizes = np.where(np.arange(330) < 200, 2.0 ** (4 - bits), 16.0)
    run(2500 + bits, lens, 4, 2, D, causal, sizes, np.ones(330), 2.0 ** 10, top_e=[200 + 64])


@pytest.mark.parametrize("D", [64, 80, 128])
def test_rows_of_different_errors(D):
    """A row's dq is its own: sizes from 2^-12 to 2^12 in one causal sequence."""
    say(f"gradients, rows of different errors, D={D}")
    rng = np.random.default_rng(2510)
    # growing errors last: no key's sum drops from a large to a small one
    run(2511, [300], 2, 1, D, True, 2.0 ** (np.arange(300) / 12.5 - 12), np.ones(300), 1.0)
    run(2512, [300], 2, 1, D, True, 2.0 ** rng.uniform(-12, 12, 300), np.ones(300), 1.0)


@pytest.mark.parametrize("D", [64, 128])
def test_values_of_different_sizes(D):
    """Values of another sequence, and of keys that a row does not see, leave
    its gradient alone."""
    say(f"gradients, values of different sizes, D={D}")
    sizes = np.where(np.arange(330) < 200, 2.0 ** -10, 1.0)
    run(2520, [200, 130], 2, 2, D, True, np.ones(330), sizes, 16.0, top_v=[199, 260])
    run(2521, [330], 2, 2, D, True, np.ones(330), 2.0 ** (np.arange(330) / 16.5 - 12), 16.0)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("fill", [0x00, TOP8, 0x7F])
def test_tokens_of_no_sequence(fill, D):
    """What lies before the first and behind the last sequence changes no bit."""
    say(f"gradients, tokens of no sequence hold {fill:#x}, D={D}")
    rng = np.random.default_rng(2530)
    T, cu = 260, np.array([37, 130, 201])
    q, k, v, e = (codes8(rng, (T, h, D), s) for h, s in ((4, 1), (2, 1), (2, 2.0 ** -8), (4, 2.0 ** -9)))
    out = (np.arange(T) < 37) | (np.arange(T) >= 201)
    want = run_attention(q[~out], k[~out], v[~out], cu - 37, cu - 37, True, 0.125, e[~out])
    for x in (q, k, v, e):
        x[out] = fill
    got = run_attention(q, k, v, cu, cu, True, 0.125, e)
    ref = lm.attention(value(q[~out]), value(k[~out]), value(v[~out]), cu - 37, cu - 37, True, 0.125,
                       value(e[~out]))
    inside = {n: (x[:, ~out] if n == "lse" else x[~out]) for n, x in got.items()}
    compare(inside, ref)
    compare(want, ref)
