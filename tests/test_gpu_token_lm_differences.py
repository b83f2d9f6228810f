"""The token model's gradient along its last norm's weights against differences in
float64: the stages behind the residual sum (norm, logits, log probabilities) are
evaluated without roundings on the sum that the model stored."""
import numpy as np
import pytest

import oracle
from paper_1812_08011_amd.token_lm import Fp8TokenLm
from tests.gpu_util import dev, host, say
from tests.lm_util import codes16, value
from tests.token_util import F32, gpu  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tau", [1.0, 2.0])
def test_last_norm_weights(tau):
    """The loss is the mean of -logp of each position's least likely token, the
    direction the weights themselves: logits z then change by z.  The model's
    gradient is off by: the probabilities of its rounded logits (measured); dZ's
    FP32 arithmetic and FP16 codes, 2^-9 of each or 2^-40 where that is less; the
    product dZ Wl^T's roundings (measured); the codes of dg2.  Together they stay
    below a twentieth of the gradient."""
    rng = np.random.default_rng(160)
    net = Fp8TokenLm([50, 14], width=64, Hq=2, Hkv=1, D=32, vocab=300)
    W = {n: oracle.fp16_quantize((1.0 + 0.2 * rng.standard_normal(s)).astype(F32)) if n in ("g1", "g2") else
         codes16(rng, s, 1.0 / np.sqrt(net.width if n == "E" else s[0])) for n, s in net.shapes.items()}
    net.set_weights(W)
    tok = dev(rng.integers(0, 300, net.T))
    net.forward(tok, dev(np.zeros((net.T, 1), np.int64)), tau)
    given = value(host(net.Z16)).argmin(1)
    scale, T, at = 1024.0, net.T, np.arange(net.T)
    net.forward(tok, dev(given[:, None]), tau)
    net.backward(tok, dev(given[:, None]), dev(np.full((T, 1), -1.0 / T, F32)), None, scale, tau)
    s1, g2, Wl = value(host(net.S1)).astype(np.float64), value(W["g2"]), value(W["Wl"])
    n = s1 / np.sqrt((s1 ** 2).mean(1, keepdims=True) + float(F32(net.eps)))

    def loss(g):
        z = (n * g) @ Wl / tau
        top = z.max(1)
        return -(z[at, given] - top - np.log(np.exp(z - top[:, None]).sum(1))).mean()
    step = 1e-4
    want = (loss(g2 * (1 + step)) - loss(g2 * (1 - step))) / (2 * step)
    dg2 = value(host(net.dW16["g2"])) / scale
    got = (dg2 * g2).sum()
    z = (n * g2) @ Wl
    softmax = lambda z: np.exp(z / tau) / np.exp(z / tau).sum(1, keepdims=True)
    p, p16 = softmax(z), softmax(value(host(net.Z16)))
    dZ = value(host(net.dZ16)) / scale
    weight = p16 + (np.arange(300) == given[:, None])          # |dz| T tau at most
    lim = ((abs(p16 - p) + 2.0 ** -9 * weight) * abs(z)).sum() / (T * tau) + 2.0 ** -40 / scale * abs(z).sum()
    lim += (abs(value(host(net.dY16)) / scale - dZ @ Wl.T) * abs(n * g2)).sum()
    lim += 2.0 ** -10 * (abs(dg2) * abs(g2)).sum()
    # the step's truncation, below step^2 / 6 of the logits' spread cubed, and 2^-50 over it
    lim += step ** 2 / 6 * (np.ptp(z, axis=1).max() / tau) ** 3 + 2.0 ** -50 * abs(loss(g2)) / step
    say("gradient", got, "differences", want, "limit", lim)
    assert lim < abs(want) / 20
    assert abs(got - want) <= lim
