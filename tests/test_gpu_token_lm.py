"""A training step of the language model from tokens to log probabilities
(paper_1812_08011_amd.token_lm): every stage against its definition on the
codes that the stage before left, and a captured step."""
import numpy as np
import pytest
import torch

import oracle
from oracle import lm
from oracle import tokens as ot
from paper_1812_08011_amd.token_lm import NAMES, Fp8TokenLm
from tests.gpu_util import dev, host, say
from tests.lm_util import check, codes16, value
from tests.token_util import F16, F32, gpu, replayed, rounded  # noqa: F401

pytestmark = pytest.mark.gpu


def model(seed, lengths, **kw):
    rng = np.random.default_rng(seed)
    net = Fp8TokenLm(lengths, **kw)
    W = {}
    for n, s in net.shapes.items():
        if n in ("g1", "g2"):
            W[n] = oracle.fp16_quantize((1.0 + 0.2 * rng.standard_normal(s)).astype(F32))
        else:
            W[n] = codes16(rng, s, 1.0 / np.sqrt(net.width if n == "E" else s[0]))
    net.set_weights(W)
    tokens = np.minimum(rng.integers(0, net.vocab, net.T), rng.integers(0, net.vocab, net.T))
    tokens[rng.random(net.T) < 0.05] = -1
    given = rng.integers(0, net.vocab, (net.T, 1))
    given[rng.random(net.T) < 0.1] = -1
    d_logp = np.full((net.T, 1), -1.0 / net.T, F32)
    return net, W, tokens, given, d_logp, np.full(net.T, -0.01 / net.T, F32)


@pytest.mark.parametrize("stream,tau", [("f32", 1.0), ("fp16", 0.7)])
def test_step_stage_by_stage(stream, tau):
    say("token language model, stage by stage", stream)
    net, W, tokens, given, d_logp, d_entropy = model(1, [37, 1, 90], width=96, Hq=4, Hkv=2, D=32, vocab=200,
                                                     top=5, stream=stream)
    S, T, CL, scale = {"f32": F32, "fp16": F16}[stream], net.T, net.CL, 1024.0
    net.step(dev(tokens), dev(given), dev(d_logp), dev(d_entropy), 0.05, 0.9, 1e-4, scale, 7, 3, tau)
    g = {n: host(getattr(net, n)).reshape(getattr(net, n).shape) for n in
         ("S0", "S1", "dS0", "dS1", "X8", "rstd1", "rstd2", "QKV16", "QKV8", "O16", "O8", "lse", "A16", "Y16",
          "Z16", "logp", "entropy", "stats", "top_idx", "top_logp", "dZ16", "dY16", "dA8", "dO8", "dQKV16",
          "dQKV8", "dX16")}
    dW = {n: host(net.dW16[n]) for n in NAMES}
    W8 = {n: oracle.fp8_quantize(W[n]) for n in ("Wqkv", "Wo")}
    flat = lambda x: np.ascontiguousarray(x.reshape(T, -1))
    f64 = lambda x: value(x).astype(np.float64)
    # embedding and the first norm
    used = (tokens >= 0)[:, None]
    s0 = np.where(used, value(W["E"][np.maximum(tokens, 0)]).astype(F32) * F32(net.scale), F32(0))
    assert np.array_equal(g["S0"], rounded(s0, S))
    eps = float(F32(net.eps))
    n1 = ot.norm(f64(g["S0"]), value(W["g1"]), eps, 1.0, False)
    check("rstd1", g["rstd1"], n1["rstd"], n1["rstd_err"])
    check("X8", g["X8"], n1["y"], n1["y_err"])
    assert np.array_equal(flat(g["QKV16"]), oracle.chunk_gemm(g["X8"], W8["Wqkv"], CL))
    # attention's own stages are the other model's; here what goes in and comes out
    q, k, v = (value(g["QKV8"][:, s]) for s in (slice(0, 4), slice(4, 6), slice(6, 8)))
    cu = host(net.cu)
    ref = lm.attention(q, k, v, cu, cu, True, float(F32(1.0 / np.sqrt(32))), value(g["dO8"]))
    check("O8", g["O8"], ref["o"], ref["o_err"])
    assert np.array_equal(g["A16"], oracle.chunk_gemm(flat(g["O8"]), W8["Wo"], CL))
    # the residual sum and the second norm
    s1 = value(g["A16"]).astype(F32) + value(g["S0"]).astype(F32)
    assert np.array_equal(g["S1"], rounded(s1, S))
    n2 = ot.norm(f64(g["S1"]), value(W["g2"]), eps, 1.0, False)
    check("Y16", g["Y16"], n2["y"], n2["y_err"])
    assert np.array_equal(g["Z16"], oracle.chunk_gemm_p16(g["Y16"], W["Wl"], CL))
    # log probabilities and the logits' gradient
    t32 = float(F32(tau))
    r = ot.logprobs(value(g["Z16"]), given, t32, 5)
    assert np.array_equal(g["top_idx"], r["top_idx"])
    for n in ("logp", "entropy", "stats", "top_logp"):
        check(n, g[n], r[n], r[n + "_err"])
    dz, dz_err = ot.logprobs_grad(value(g["Z16"]), given, t32, f64(g["stats"]), f64(g["entropy"]),
                                  f64(d_logp), f64(d_entropy), scale)
    check("dZ16", g["dZ16"], dz, dz_err)
    assert np.array_equal(g["dY16"], oracle.chunk_gemm_p16(g["dZ16"], W["Wl"], CL, 0, 1))
    assert np.array_equal(dW["Wl"], oracle.chunk_gemm_p16(g["Y16"], g["dZ16"], CL, 1, 0))
    d, err, dg, dg_err = ot.norm_grad(f64(g["S1"]), value(W["g2"]), f64(g["rstd2"]), value(g["dY16"]), None)
    check("dS1", g["dS1"], d, err)
    check("dA8", g["dA8"], d, err + abs(d) * 2.0 ** -23)
    check("g2", dW["g2"], dg, dg_err)
    assert np.array_equal(dW["Wo"], oracle.chunk_gemm(flat(g["O8"]), g["dA8"], CL, 1, 0))
    assert np.array_equal(flat(g["dO8"]), oracle.fp8_quantize(oracle.chunk_gemm(g["dA8"], W8["Wo"], CL, 0, 1)))
    for n, s in (("dq", slice(0, 4)), ("dk", slice(4, 6)), ("dv", slice(6, 8))):
        check(n, g["dQKV16"][:, s], ref[n], ref[n + "_err"])
    assert np.array_equal(dW["Wqkv"], oracle.chunk_gemm(g["X8"], flat(g["dQKV8"]), CL, 1, 0))
    assert np.array_equal(g["dX16"], oracle.chunk_gemm(flat(g["dQKV8"]), W8["Wqkv"], CL, 0, 1))
    d, err, dg, dg_err = ot.norm_grad(f64(g["S0"]), value(W["g1"]), f64(g["rstd1"]), value(g["dX16"]),
                                      f64(g["dS1"]))
    check("dS0", g["dS0"], d, err)
    check("g1", dW["g1"], dg, dg_err)
    de, de_err = ot.embed_grad(tokens, value(g["dS0"]), net.vocab, float(F32(net.scale)))
    check("E", dW["E"], de, de_err + 2 * abs(de) * 2.0 ** -24)
    # updates
    lr, wd = float(F32(0.05) / F32(scale)), float(F32(1e-4) * F32(scale))
    for i, n in enumerate(NAMES):
        w, m, w8 = oracle.sr_weight_update(W[n].ravel(), dW[n].ravel(), np.zeros(W[n].size, np.uint16), lr=lr,
                                           momentum=0.9, weight_decay=0.0 if n in ("g1", "g2") else wd, seed=7,
                                           offset=3 * 6 + i)
        assert np.array_equal(host(net.W16[n]).ravel(), w), n
        assert np.array_equal(host(net.V16[n]).ravel(), m), n
        if n in net.W8:
            assert np.array_equal(host(net.W8[n]).ravel(), w8), n


def test_gradients_follow_differences():
    """<gradient, direction> of the mean of -logp against differences along a
    direction of the last norm's weights, in the last stages that are smooth (FP16
    operands): their rounding, 2^-10 of each of width products, and the step's
    truncation, over the step."""
    net, W, tokens, given, d_logp, _ = model(2, [50, 14], width=64, Hq=2, Hkv=1, D=32, vocab=300)
    tok, giv = dev(tokens), dev(given)
    weight = float((given >= 0).sum()) / net.T
    loss = lambda: -float(host(net.forward(tok, giv)).astype(np.float64).sum()) / net.T
    net.set_weights(W)
    loss()
    net.backward(tok, giv, dev(d_logp), None, 1024.0)
    grad = value(host(net.dW16["g2"])) / 1024.0
    step = 2.0 ** -3
    up, down = dict(W), dict(W)
    up["g2"] = oracle.fp16_quantize((value(W["g2"]) * (1 + step)).astype(F32))
    down["g2"] = oracle.fp16_quantize((value(W["g2"]) * (1 - step)).astype(F32))
    net.set_weights(up)
    a = loss()
    net.set_weights(down)
    b = loss()
    want = (grad * (value(up["g2"]) - value(down["g2"]))).sum()
    net.set_weights(W)
    net.forward(tok, giv)
    z = value(host(net.Z16))
    spread = z.max(1) - z.min(1)
    # logits move by at most step times themselves: the third derivative of a log
    # probability along them is below spread^3; the codes' roundings are 2^-9
    lim = weight * ((step * spread.max()) ** 3 / 3 + 2 * 2.0 ** -9 * spread.max())
    say("difference", a - b, "gradient", want, "limit", lim)
    assert abs((a - b) - want) <= lim
    assert abs(want) > 0


def test_captured_step():
    net, W, tokens, given, d_logp, d_entropy = model(3, [40, 25], width=64, Hq=2, Hkv=1, D=32, vocab=300)
    args = dev(tokens), dev(given)
    dl, dh = dev(d_logp), dev(d_entropy)

    def call():
        net.forward(*args)
        net.backward(*args, dl, dh, 1024.0)
    replayed(call, [net.logp, net.entropy, net.dS0, *net.dW16.values()])


def test_empty_batch():
    net = Fp8TokenLm([], width=64, Hq=2, Hkv=1, D=32, vocab=100)
    i64 = lambda *s: torch.zeros(s, dtype=torch.int64, device=net.dev)
    net.forward(i64(0), i64(0, 1))
    for n in NAMES:
        net.dW16[n].view(torch.int16).fill_(5)
    net.backward(i64(0), i64(0, 1), torch.zeros(0, 1, device=net.dev), None, 1.0)
    for n in ("E", "g1", "g2"):
        assert (host(net.dW16[n]) == 0).all(), n
