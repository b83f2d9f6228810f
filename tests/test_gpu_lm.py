"""A training step of the small language model (paper_1812_08011_amd.lm): every
stage against its definition on the codes that the stage before left, and the
loss over some steps on one batch."""
import numpy as np
import pytest
import torch

import oracle
import paper_1812_08011_amd as fp8t
from oracle import lm
from oracle import mlp as omlp
from paper_1812_08011_amd.lm import Fp8AttentionLm
from tests.gpu_util import dev, host, say
from tests.lm_util import check, codes8, value

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    fp8t.lib()
    yield


def model(seed, lengths, **kw):
    rng = np.random.default_rng(seed)
    net = Fp8AttentionLm(lengths, **kw)
    W = [oracle.fp16_quantize((rng.standard_normal(s) / np.sqrt(s[0])).astype(np.float32))
         for s in net.shapes]
    net.set_weights(W)
    X8 = codes8(rng, (net.T, net.width))
    k = 6
    idx = np.stack([rng.choice(net.vocab, k, replace=False) for _ in range(net.T)]).astype(np.int64)
    idx[rng.random(idx.shape) < 0.1] = -1
    t = (rng.standard_normal((net.T, k)) * 2).astype(np.float32)
    w = np.where(rng.random(net.T) < 0.1, 0.0, 1.0 / net.T).astype(np.float32)
    return net, W, X8, idx, t, w


def test_step_stage_by_stage():
    say("language model step, stage by stage")
    lengths = [37, 1, 90]
    net, W, X8, idx, t, w = model(1, lengths, width=96, Hq=4, Hkv=2, D=32, hidden=80, vocab=200)
    scale, T, H, D = 1024.0, net.T, net.Hq + 2 * net.Hkv, net.D
    net.step(dev(X8), dev(idx), dev(t), dev(w), 2.0, 0.05, 0.9, 1e-4, scale, 7, 0)
    got = {n: host(getattr(net, n)).reshape(getattr(net, n).shape) for n in
           ("QKV16", "QKV8", "O16", "O8", "lse", "H16", "A16", "Y16", "loss", "E16", "dA16", "E8", "dO8",
            "dQKV16", "dQKV8")}
    W8 = [oracle.fp8_quantize(x) for x in W[:2]]
    flat = lambda x: np.ascontiguousarray(x.reshape(T, -1))
    assert np.array_equal(flat(got["QKV16"]), oracle.chunk_gemm(X8, W8[0], net.CL))
    turned, pos, freqs = net.Hq + net.Hkv, host(net.positions), host(net.freqs)
    x = value(got["QKV16"])
    want = lm.rotary(x[:, :turned], pos, freqs)
    check("rotary", got["QKV8"][:, :turned], want, 2e-6 * (abs(want) + np.sqrt((x ** 2).sum(-1, keepdims=True))[:, :turned]))
    assert np.array_equal(got["QKV8"][:, turned:], oracle.fp8_quantize(got["QKV16"][:, turned:]))
    q, k, v = (value(got["QKV8"][:, s]) for s in (slice(0, net.Hq), slice(net.Hq, turned), slice(turned, H)))
    cu = host(net.cu)
    c = float(np.float32(1.0 / np.sqrt(D)))
    ref = lm.attention(q, k, v, cu, cu, True, c, value(got["dO8"]))
    for n, g in (("o", got["O16"]), ("o", got["O8"]), ("lse", got["lse"])):
        check(n, g, ref[n], ref[n + "_err"])
    assert np.array_equal(got["H16"], oracle.chunk_gemm(flat(got["O8"]), W8[1], net.CL))
    assert np.array_equal(got["A16"], omlp.relu16(got["H16"]))
    assert np.array_equal(got["Y16"], oracle.chunk_gemm_p16(got["A16"], W[2], net.CL))
    loss, g, loss_err, g_err = lm.distill(value(got["Y16"]), idx, t.astype(np.float64), w.astype(np.float64),
                                          2.0, scale)
    check("loss", got["loss"], loss, loss_err)
    check("E16", got["E16"], g, g_err)
    assert np.array_equal(got["dA16"], oracle.chunk_gemm_p16(got["E16"], W[2], net.CL, 0, 1))
    assert np.array_equal(got["E8"], omlp.relu_backward_fp8(got["dA16"], got["H16"], 1.0))
    do16 = oracle.chunk_gemm(got["E8"], W8[1], net.CL, 0, 1)
    assert np.array_equal(flat(got["dO8"]), oracle.fp8_quantize(do16))
    d = got["dQKV16"]
    for n, s in (("dq", slice(0, net.Hq)), ("dk", slice(net.Hq, turned)), ("dv", slice(turned, H))):
        check(n, d[:, s], ref[n], ref[n + "_err"])
    x = value(d)
    want = lm.rotary(x[:, :turned], pos, freqs, inverse=True)
    check("inverse", got["dQKV8"][:, :turned], want, 2e-6 * (abs(want) + np.sqrt((x ** 2).sum(-1, keepdims=True))[:, :turned]))
    assert np.array_equal(got["dQKV8"][:, turned:], oracle.fp8_quantize(d[:, turned:]))
    dW = [oracle.chunk_gemm(X8, flat(got["dQKV8"]), net.CL, 1, 0),
          oracle.chunk_gemm(flat(got["O8"]), got["E8"], net.CL, 1, 0),
          oracle.chunk_gemm_p16(got["A16"], got["E16"], net.CL, 1, 0)]
    for i in range(3):
        assert np.array_equal(host(net.dW16[i]), dW[i]), i
        lr = float(np.float32(0.05) / np.float32(scale))
        wd = float(np.float32(1e-4) * np.float32(scale))
        nw, nv, n8 = oracle.sr_weight_update(W[i].ravel(), dW[i].ravel(), np.zeros(W[i].size, np.uint16),
                                             lr=lr, momentum=0.9, weight_decay=wd, seed=7, offset=i)
        assert np.array_equal(host(net.W16[i]).ravel(), nw), i
        assert np.array_equal(host(net.V16[i]).ravel(), nv), i
        if i < 2:
            assert np.array_equal(host(net.W8[i]).ravel(), n8), i


def test_the_loss_falls():
    say("language model, twenty steps")
    net, W, X8, idx, t, w = model(2, [64, 200, 33], width=128, Hq=4, Hkv=1, D=64, hidden=128, vocab=500)
    args = (dev(X8), dev(idx), dev(t), dev(w))
    losses = [float(net.step(*args, 1.0, 0.5, 0.9, 0.0, 1024.0, 3, s).sum()) for s in range(20)]
    assert np.isfinite(losses).all() and losses[-1] < 0.7 * losses[0], losses
