"""Measured cases of the operators at both ends of a language model and at its
joints: token embeddings with their gradient, the norm of a residual sum with
its gradient, and the log probabilities of given tokens with theirs.

``run`` makes one pass: with ``own`` true through the package's public
functions, with ``own`` false in elementary torch operations in 32 bits (long
sums in 64), rounded once at the end.

Formats: FP8 (1,5,2) codes in uint8 are torch's float8_e5m2 bit for bit and
come back as that type.  FP16 (1,6,9) codes in uint16 have no torch type; a
result in FP16 comes back as IEEE half, which holds every FP16 value from 2^-14
to 2^16 exactly (fp16_dequantize).

Kinds:

* ``embed``      -- rows of a table by tokens, scaled.
* ``embed_grad`` -- the table's gradient: errors summed by token, every row written.
* ``norm``       -- h = x + r, y = h / rms(h) w, with each row's own scale or one.
* ``norm_grad``  -- the gradients of h (in two formats) and of w.
* ``logp``       -- log probabilities of given tokens, entropy, the k likeliest tokens.
* ``logp_grad``  -- the logits' gradient from those of the log probabilities and the entropy.
"""
import math

import torch

own = False
DEV = "cuda:0"


def listed():
    return [
        # the token that a step of generation starts from
        dict(name="embed_token", kind="embed", T=1, V=32768, W=1024, table="fp16", out="fp8",
             scale=32.0),
        # a packed training batch into a residual stream in 32 bits, odd vocabulary
        dict(name="embed_batch", kind="embed", T=16384, V=50001, W=2048, table="fp16", out="f32",
             scale=45.25),
        # a small model's step (vocabulary 1024, width 256), gradient for the FP16 update
        dict(name="embed_grad_small", kind="embed_grad", T=257, V=1024, W=256, e="fp16", g="fp16",
             scale=16.0),
        # a training batch of text: few tokens make up most of it, most rows get nothing
        dict(name="embed_grad_batch", kind="embed_grad", T=16384, V=32768, W=1024, e="fp16",
             g="f32", scale=32.0),
        # one token between two GEMMs of a step of generation
        dict(name="norm_token", kind="norm", T=1, W=1024, x="fp16", r="f32", w="fp16", y="fp8",
             eps=1e-5, rows=False),
        # a long batch, the residual stream in 32 bits, each row of the GEMM's operand scaled
        dict(name="norm_batch", kind="norm", T=16384, W=4096, x="fp16", r="f32", w="fp16", y="fp8",
             eps=1e-5, rows=True),
        # backward through a norm of odd width, everything in the training formats
        dict(name="norm_grad_odd", kind="norm_grad", T=5003, W=1001, h="fp16", w="fp16", dy="fp8",
             d="fp16", dw="fp16", residual=False, eps=1e-6),
        # a long batch: the error from above joins, the GEMM below gets its own in FP8
        dict(name="norm_grad_batch", kind="norm_grad", T=8192, W=4096, h="f32", w="fp16",
             dy="fp16", d="f32", dw="f32", residual=True, eps=1e-5),
        # the next token of one sequence, part of the vocabulary masked out
        dict(name="logp_token", kind="logp", N=1, V=50001, z="f32", m=1, k=20, tau=1.0,
             masked=True),
        # a teacher's logits over a batch: the entries that a distillation keeps
        dict(name="logp_vocab", kind="logp", N=4096, V=32768, z="fp16", m=1, k=64, tau=1.0,
             masked=False),
        # several given tokens for each row, odd sizes, a temperature
        dict(name="logp_grad_odd", kind="logp_grad", N=777, V=50001, z="f32", m=3, tau=2.0,
             entropy=True, g="f32"),
        # a policy's update: weighted tokens and an entropy term, the error in FP8
        dict(name="logp_grad_vocab", kind="logp_grad", N=4096, V=32768, z="fp16", m=1, tau=1.0,
             entropy=True, g="fp8"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def _draw_embed(rng):
    W = _log_int(rng, 32, 4096)
    V = _log_int(rng, 100, min(131072, 2 ** 27 // W))
    return dict(kind="embed", T=_log_int(rng, 1, 2 ** 25 // W), V=V, W=W,
                table=rng.choice(["fp16", "fp16", "fp8", "f32"]),
                out=rng.choice(["fp8", "fp16", "f32"]), scale=rng.choice([1.0, math.sqrt(W)]))


def _draw_embed_grad(rng):
    W = _log_int(rng, 32, 4096)
    V = _log_int(rng, 100, min(131072, 2 ** 26 // W))
    return dict(kind="embed_grad", T=_log_int(rng, 1, min(65536, 2 ** 25 // W)), V=V, W=W,
                e=rng.choice(["fp8", "fp16", "fp16", "f32"]), g=rng.choice(["fp16", "f32", "f32"]),
                scale=rng.choice([1.0, math.sqrt(W)]))


def _draw_norm(rng):
    W = _log_int(rng, 32, 16384)
    return dict(kind="norm", T=_log_int(rng, 1, min(32768, 2 ** 26 // W)), W=W,
                x=rng.choice(["fp16", "fp16", "f32"]), r=rng.choice(["f32", "f32", "fp16", ""]),
                w=rng.choice(["fp16", "f32"]), y=rng.choice(["fp8", "fp8", "fp16"]),
                eps=rng.choice([1e-5, 1e-6]), rows=rng.random() < 0.4)


def _draw_norm_grad(rng):
    W = _log_int(rng, 32, 16384)
    return dict(kind="norm_grad", T=_log_int(rng, 1, min(32768, 2 ** 25 // W)), W=W,
                h=rng.choice(["f32", "fp16"]), w=rng.choice(["fp16", "f32"]),
                dy=rng.choice(["fp8", "fp16", "f32"]), d=rng.choice(["f32", "fp16"]),
                dw=rng.choice(["f32", "fp16"]), residual=rng.random() < 0.7,
                eps=rng.choice([1e-5, 1e-6]))


def _draw_logp(rng):
    V = _log_int(rng, 300, 131072)
    return dict(kind="logp", N=_log_int(rng, 1, min(8192, 2 ** 26 // V)), V=V,
                z=rng.choice(["fp16", "f32"]), m=rng.choice([1, 1, 3, 8]),
                k=rng.choice([0, 1, 5, 20, 64, 100]), tau=rng.choice([1.0, 1.0, 0.7, 2.0]),
                masked=rng.random() < 0.4)


def _draw_logp_grad(rng):
    V = _log_int(rng, 300, 131072)
    z = rng.choice(["fp16", "f32"])
    return dict(kind="logp_grad", N=_log_int(rng, 1, min(8192, 2 ** 26 // V)), V=V, z=z,
                m=rng.choice([1, 1, 3, 8]), tau=rng.choice([1.0, 1.0, 0.7, 2.0]),
                entropy=rng.random() < 0.6,
                g=rng.choice(["fp16", "fp8"]) if z == "fp16" else "f32")


def draw(rng):
    return rng.choice([_draw_embed, _draw_embed_grad, _draw_embed_grad, _draw_norm, _draw_norm_grad,
                       _draw_logp, _draw_logp_grad])(rng)


# ---- the storage formats in torch operations ----------------------------------------

def _round16(x):
    """float32 -> nearest FP16 (1,6,9) value, ties to even, as float32."""
    u = x.view(torch.int32)
    r = ((u + 0x1FFF + ((u >> 14) & 1)) & ~0x3FFF).view(torch.float32)
    low = torch.round(x * 2.0 ** 39) * 2.0 ** -39          # below 2^-30 the step is 2^-39
    return torch.where(x.abs() < 2.0 ** -30, low, r)


def _encode16(x):
    """float32 -> FP16 codes (uint16), for values below 2^32 and infinities."""
    r = _round16(x)
    u = r.view(torch.int32) & 0x7FFFFFFF
    code = torch.where(r.abs() < 2.0 ** -30, (r.abs() * 2.0 ** 39).to(torch.int32),
                       (u >> 14) - (96 << 9))
    code = torch.where(r.isinf(), 0x7E00, code)
    code = code | torch.where(r < 0, 0x8000, 0).to(torch.int32)
    return code.to(torch.int16).view(torch.uint16)


def _decode16(c):
    """FP16 codes -> float32: exponent and significand moved into float32's
    fields, the exponents' bias (127 - 31) restored by a product."""
    i = c.view(torch.int16).to(torch.int32)
    x = ((i << 14) & -1610612737).view(torch.float32) * 2.0 ** 96
    return torch.where(x.abs() >= 2.0 ** 32, x * math.inf, x)


def _encode8(x):
    return x.clamp(-57344.0, 57344.0).to(torch.float8_e5m2)


def _plain(c):
    """Codes or floats -> float32."""
    return c if c.dtype == torch.float32 else _decode16(c) if c.dtype == torch.uint16 else \
        c.view(torch.float8_e5m2).to(torch.float32)


def _as(x, out):
    """float32 results in the storage type `out`, as the values that come back."""
    return x if out == "f32" else _encode8(x) if out == "fp8" else _round16(x).to(torch.float16)


_BYTES = {"f32": 4, "fp16": 2, "fp8": 1, "": 0}
_DTYPE = {"f32": torch.float32, "fp16": torch.uint16, "fp8": torch.uint8}


def _buffer(out, *shape):
    return torch.empty(shape, dtype=_DTYPE[out], device=DEV)


def _results(s, **formats):
    """Room for the results of a pass, and for the values of those in FP16."""
    for n, (out, shape) in formats.items():
        s[n] = _buffer(out, *shape)
        if out == "fp16":
            s[n + "_half"] = torch.empty(shape, dtype=torch.float16, device=DEV)


def _values(s, n):
    """A result as values: FP16 codes through the package's decoder."""
    if s[n].dtype != torch.uint16:
        return s[n].view(torch.float8_e5m2) if s[n].dtype == torch.uint8 else s[n]
    import paper_1812_08011_amd as fp8t
    return fp8t.fp16_dequantize(s[n], s[n + "_half"])


# ---- inputs ---------------------------------------------------------------------------

def _normal(gen, shape, std=1.0):
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32) * std


def _take(codes, at):
    """Rows of an array of codes or floats."""
    return codes.view(torch.int16)[at].view(torch.uint16) if codes.dtype == torch.uint16 else codes[at]


def _stored(x, fmt):
    return x.contiguous() if fmt == "f32" else _encode16(x) if fmt == "fp16" else \
        _encode8(x).view(torch.uint8)


def _tokens(gen, T, V):
    """Tokens as text has them: the r-th most frequent one with a probability of
    log((r + 2) / (r + 1)) / log(V + 1), its number anywhere; one in 64 is none."""
    u = torch.rand((T,), generator=gen, device=DEV, dtype=torch.float64)
    rank = ((V + 1.0) ** u).to(torch.int64).clamp(1, V) - 1
    none = torch.rand((T,), generator=gen, device=DEV) < 1.0 / 64.0
    return torch.where(none, -1, rank * 7919 % V)


def _prepare_embed(c, gen):
    s = dict(c, tokens=_tokens(gen, c["T"], c["V"]))
    s["table"] = _stored(_normal(gen, (c["V"], c["W"]), 0.02), c["table"])
    _results(s, y=(c["out"], (c["T"], c["W"])))
    return s


def _prepare_embed_grad(c, gen):
    s = dict(c, tokens=_tokens(gen, c["T"], c["V"]), ws={})
    # the error of the first layer's input under a loss scale of 1024
    s["e"] = _stored(_normal(gen, (c["T"], c["W"]), 1e-3) * 1024.0, c["e"])
    _results(s, g_out=(c["g"], (c["V"], c["W"])))
    return s


def _stream(gen, T, W):
    """A residual stream: some channels much larger than the others."""
    x = _normal(gen, (T, W), 2.0)
    return x * torch.exp(_normal(gen, (W,), 0.5))


def _weight(gen, W, fmt):
    return _stored(1.0 + _normal(gen, (W,), 0.2), fmt)


def _prepare_norm(c, gen):
    T, W = c["T"], c["W"]
    s = dict(c, r_format=c["r"])
    s["x"] = _stored(_normal(gen, (T, W)), c["x"])
    s["r"] = _stored(_stream(gen, T, W), c["r"]) if c["r"] else None
    s["w"] = _weight(gen, W, c["w"])
    if c["r"]:
        _results(s, h=(c["r"], (T, W)))
    _results(s, y_out=(c["y"], (T, W)), rstd=("f32", (T,)), scales=("f32", (T,)))
    return s


def _prepare_norm_grad(c, gen):
    T, W = c["T"], c["W"]
    s = dict(c, ws={})
    s["h"] = _stored(_stream(gen, T, W), c["h"])
    s["w"] = _weight(gen, W, c["w"])
    s["rstd"] = torch.rsqrt(_plain(s["h"]).double().square().mean(1) + c["eps"]).float()
    s["dy"] = _stored(_normal(gen, (T, W), 1e-3) * 1024.0, c["dy"])
    s["dr"] = _stored(_normal(gen, (T, W), 1e-3) * 1024.0, c["d"]) if c["residual"] else None
    _results(s, dx=(c["d"], (T, W)), dx8=("fp8", (T, W)), dw_out=(c["dw"], (W,)))
    return s


def _logits(gen, c, masked):
    """Logits, and m given tokens for each row: likely ones, some of them none."""
    N, V, m = c["N"], c["V"], c["m"]
    z = _normal(gen, (N, V), 2.0)
    idx = torch.randint(0, V, (N, m), generator=gen, device=DEV)
    z.scatter_add_(1, idx, 4.0 + _normal(gen, (N, m)))
    if masked:                          # a part of the vocabulary that may not follow
        z.masked_fill_(torch.rand((N, V), generator=gen, device=DEV) < 0.3, -math.inf)
    if m > 1:
        none = torch.rand((N, m), generator=gen, device=DEV) < 0.2
        idx = torch.where(none, -1, idx)
    return _stored(z, c["z"]), idx


def _prepare_logp(c, gen):
    N, k = c["N"], c["k"]
    s = dict(c, ws={})
    s["z"], s["idx"] = _logits(gen, c, c["masked"])
    _results(s, logp=("f32", (N, c["m"])), entropy=("f32", (N,)), stats=("f32", (N, 2)),
             top_logp=("f32", (N, k)))
    s["top_idx"] = torch.empty((N, k), dtype=torch.int64, device=DEV)
    return s


def _prepare_logp_grad(c, gen):
    N, m = c["N"], c["m"]
    s = dict(c)
    s["z"], s["idx"] = _logits(gen, c, False)
    # what the forward pass left
    s["stats"], s["entropy_of"] = torch.empty((N, 2), device=DEV), torch.empty((N,), device=DEV)
    for r in range(0, N, 512):
        x = _plain(s["z"][r:r + 512]).double()
        top = x.amax(1)
        d = (x - top[:, None]) / c["tau"]
        ls = torch.log(torch.exp(d).sum(1))
        s["stats"][r:r + 512, 0], s["stats"][r:r + 512, 1] = top, ls
        s["entropy_of"][r:r + 512] = ls - (torch.softmax(d, 1) * d).sum(1)
    s["d_logp"] = _normal(gen, (N, m)) / N
    s["d_entropy"] = torch.full((N,), 0.01 / N, device=DEV) if c["entropy"] else None
    s["grad_scale"] = 1024.0 * N
    _results(s, g_out=(c["g"], (N, c["V"])))
    return s


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return {"embed": _prepare_embed, "embed_grad": _prepare_embed_grad, "norm": _prepare_norm,
            "norm_grad": _prepare_norm_grad, "logp": _prepare_logp,
            "logp_grad": _prepare_logp_grad}[case["kind"]](case, gen)


# ---- one pass through the framework -----------------------------------------------------

def _workspace(s, size):
    """A program keeps its workspace."""
    if "bytes" not in s["ws"]:
        n = s["ws"]["bytes"] = size()
        s["ws"]["buffer"] = torch.empty(n, dtype=torch.uint8, device=DEV) if n else None
    return s["ws"]["buffer"], s["ws"]["bytes"]


def _own_embed(s):
    import paper_1812_08011_amd as fp8t
    fp8t.embed_fwd(s["tokens"], s["table"], s["y"], s["scale"])
    return {"y": _values(s, "y")}


def _own_embed_grad(s):
    import paper_1812_08011_amd as fp8t
    ws = _workspace(s, lambda: fp8t.embed_bwd_workspace_size(s["tokens"], s["e"], s["g_out"]))
    fp8t.embed_bwd(s["tokens"], s["e"], s["g_out"], s["scale"], *ws)
    return {"g": _values(s, "g_out")}


def _own_norm(s):
    import paper_1812_08011_amd as fp8t
    # each row's largest result to 28672 with a scale of its own, or all times 1
    fp8t.rms_norm_fwd(s["x"], s["r"], s["w"], s["eps"], s.get("h"), s["y_out"],
                      y_scale=28672.0 if s["rows"] else 1.0,
                      y_row_scale=s["scales"] if s["rows"] else None, rstd=s["rstd"])
    out = {"y": _values(s, "y_out"), "rstd": s["rstd"]}
    if s["r"] is not None:
        out["h"] = _values(s, "h")
    if s["rows"]:
        out["scales"] = s["scales"]
    return out


def _own_norm_grad(s):
    import paper_1812_08011_amd as fp8t
    ws = _workspace(s, lambda: fp8t.rms_norm_bwd_workspace_size(s["h"]))
    fp8t.rms_norm_bwd(s["h"], s["w"], s["rstd"], s["dy"], s["dr"], s["dx"], s["dx8"], 1.0,
                      s["dw_out"], *ws)
    return {"dx": _values(s, "dx"), "dx8": _values(s, "dx8"), "dw": _values(s, "dw_out")}


def _own_logp(s):
    import paper_1812_08011_amd as fp8t
    ws = _workspace(s, lambda: fp8t.token_logprobs_workspace_size(s["z"], s["k"]))
    fp8t.token_logprobs(s["z"], s["idx"], s["tau"], s["logp"], s["entropy"], s["stats"],
                        s["top_idx"], s["top_logp"], *ws)
    return {n: s[n] for n in ("logp", "entropy", "stats", "top_idx", "top_logp")}


def _own_logp_grad(s):
    import paper_1812_08011_amd as fp8t
    fp8t.token_logprobs_bwd(s["z"], s["idx"], s["tau"], s["stats"], s["entropy_of"], s["d_logp"],
                            s["d_entropy"], s["grad_scale"], s["g_out"])
    return {"g": _values(s, "g_out")}


# ---- the same in elementary torch operations ----------------------------------------------

def _plain_embed(s):
    used = s["tokens"] >= 0
    rows = _plain(_take(s["table"], s["tokens"].clamp(min=0))) * s["scale"]
    return {"y": _as(torch.where(used[:, None], rows, 0.0), s["out"])}


def _plain_embed_grad(s):
    # one row more for what belongs to no token; sums of many errors in 64 bits
    g = torch.zeros((s["V"] + 1, s["W"]), dtype=torch.float64, device=DEV)
    at = torch.where(s["tokens"] >= 0, s["tokens"], s["V"])
    g.index_add_(0, at, _plain(s["e"]).double())
    return {"g": _as((g[:-1] * s["scale"]).float(), s["g"])}


def _plain_norm(s):
    u, out = _plain(s["x"]), {}
    if s["r"] is not None:
        u = u + _plain(s["r"])
        out["h"] = _as(u, s["r_format"])
        if s["r_format"] == "fp16":                        # the norm is of what is stored
            u = _round16(u)
    rstd = torch.rsqrt(u.double().square().mean(1) + s["eps"]).float()
    y = u * rstd[:, None] * _plain(s["w"])
    if s["rows"]:
        top = y.abs().amax(1)
        out["scales"] = torch.where(top > 0.0, 28672.0 / top, 1.0)
        y = y * out["scales"][:, None]
    out["y"], out["rstd"] = _as(y, s["y"]), rstd
    return out


def _plain_norm_grad(s):
    h, dy, rstd = _plain(s["h"]), _plain(s["dy"]), s["rstd"][:, None]
    n, wdy = h * rstd, dy * _plain(s["w"])
    dx = (wdy - n * (n * wdy).double().mean(1, keepdim=True).float()) * rstd
    if s["dr"] is not None:
        dx = dx + _plain(s["dr"])
    dw = (n * dy).double().sum(0).float()
    return {"dx": _as(dx, s["d"]), "dx8": _as(dx, "fp8"), "dw": _as(dw, s["dw"])}


def _order(z):
    """Whole numbers ordered as the logits are, among equals the lowest index first."""
    i = (z.view(torch.int16) if z.dtype == torch.uint16 else z.view(torch.int32)).to(torch.int64)
    low = -(1 << (15 if z.dtype == torch.uint16 else 31))
    i = torch.where(i < 0, low - i, i)                     # -0 is 0
    return i * (1 << 31) + ((1 << 31) - 1 - torch.arange(z.shape[1], device=DEV))


def _plain_logp(s):
    z = _plain(s["z"])
    top = z.amax(1, keepdim=True)
    d = (z - top) / s["tau"]
    e = torch.exp(d)
    l = e.sum(1, keepdim=True)
    ls = torch.log(l)
    entropy = ls[:, 0] - (torch.where(e > 0.0, d, 0.0).mul_(e)).sum(1) / l[:, 0]
    idx = s["idx"]
    logp = torch.where(idx >= 0, torch.gather(d, 1, idx.clamp(min=0)) - ls, 0.0)
    at = torch.topk(_order(s["z"]), s["k"], dim=1).indices
    return {"logp": logp, "entropy": entropy, "stats": torch.cat([top, ls], 1), "top_idx": at,
            "top_logp": torch.gather(d, 1, at) - ls}


def _plain_logp_grad(s):
    used, at = s["idx"] >= 0, s["idx"].clamp(min=0)
    logp = (_plain(s["z"]) - s["stats"][:, :1]) / s["tau"] - s["stats"][:, 1:]
    p, dl = torch.exp(logp), torch.where(used, s["d_logp"], 0.0)
    f = dl.sum(1, keepdim=True)
    if s["d_entropy"] is not None:
        f = f + s["d_entropy"][:, None] * (logp + s["entropy_of"][:, None])
    g = (-p * f).scatter_add_(1, at, dl)
    return {"g": _as(g * (s["grad_scale"] / s["tau"]), s["g"])}


def run(state):
    if own:
        return {"embed": _own_embed, "embed_grad": _own_embed_grad, "norm": _own_norm,
                "norm_grad": _own_norm_grad, "logp": _own_logp,
                "logp_grad": _own_logp_grad}[state["kind"]](state)
    return {"embed": _plain_embed, "embed_grad": _plain_embed_grad, "norm": _plain_norm,
            "norm_grad": _plain_norm_grad, "logp": _plain_logp,
            "logp_grad": _plain_logp_grad}[state["kind"]](state)


# ---- the definitions in 64 bits -----------------------------------------------------------

def _f64(c):
    """Codes (or float32) -> float64, from the fields of the format."""
    if c.dtype == torch.float32:
        return c.double()
    eb, mb = (5, 2) if c.dtype == torch.uint8 else (6, 9)
    i = c.to(torch.int64) if c.dtype == torch.uint8 else c.view(torch.int16).to(torch.int64) & 0xFFFF
    e, m = (i >> mb) & (2 ** eb - 1), (i & (2 ** mb - 1)).double()
    bias = 2 ** (eb - 1) - 1
    one = torch.ones((), dtype=torch.float64, device=c.device)
    mag = torch.where(e == 0, m * 2.0 ** (1 - bias - mb),
                      torch.ldexp(one + m * 2.0 ** -mb, (e - bias).double()))
    mag = torch.where(e == 2 ** eb - 1, math.inf, mag)
    return torch.where((i >> (eb + mb)) & 1 == 1, -mag, mag)


def _to_step(x, bits, low):
    """float64 -> `bits` bits of significand, a step of 2^low at least, ties to even."""
    step = torch.ldexp(torch.ones_like(x), (torch.frexp(x)[1] - bits).clamp(min=low).double())
    return torch.round(x / step) * step


def _in(x, fmt):
    """What a storage format makes of float64 results (FP8: three bits, to 57344)."""
    return x if fmt == "f32" else _to_step(x, 10, -39) if fmt == "fp16" else \
        _to_step(x, 3, -16).clamp(-57344.0, 57344.0)


def _exact_embed(c, s):
    t = s["tokens"].clamp(min=0)
    y = _f64(_take(s["table"], t)) * c["scale"] * (s["tokens"] >= 0)[:, None]
    return {"y": _in(y, c["out"])}


def _exact_embed_grad(c, s):
    """Running sums of the errors in the tokens' order: a row's gradient is the
    difference of two of them."""
    order = torch.argsort(s["tokens"], stable=True)
    sums = torch.cumsum(_f64(_take(s["e"], order)), 0)
    sums = torch.cat([torch.zeros_like(sums[:1]), sums])
    at = torch.searchsorted(s["tokens"][order].contiguous(), torch.arange(c["V"] + 1, device=DEV))
    return {"g": _in((sums[at[1:]] - sums[at[:-1]]) * c["scale"], c["g"])}


def _exact_norm(c, s):
    u, out = _f64(s["x"]), {}
    if s["r"] is not None:
        u = out["h"] = _in(u + _f64(s["r"]), c["r"])       # the norm is of what is stored
    rstd = out["rstd"] = (u.square().mean(1) + c["eps"]) ** -0.5
    y = u * rstd[:, None] * _f64(s["w"])
    if c["rows"]:
        out["scales"] = 28672.0 / y.abs().amax(1)
        y = y * out["scales"][:, None]
    out["y"] = _in(y, c["y"])
    return out


def _exact_norm_grad(c, s):
    h, dy, r, w = _f64(s["h"]), _f64(s["dy"]), s["rstd"].double(), _f64(s["w"])
    inner = ((h * dy) @ w) / c["W"]
    dx = r[:, None] * dy * w - (r ** 3 * inner)[:, None] * h
    if s["dr"] is not None:
        dx += _f64(s["dr"])
    return {"dx": _in(dx, c["d"]), "dx8": _in(dx, "fp8"), "dw": _in(r @ (h * dy), c["dw"])}


def _exact_logp(c, s):
    out = {n: [] for n in ("logp", "entropy", "stats", "top_logp")}
    for r in range(0, c["N"], 256):
        x, idx = _f64(s["z"][r:r + 256]), s["idx"][r:r + 256]
        lp = torch.log_softmax(x / c["tau"], 1)
        top = x.amax(1)
        out["stats"].append(torch.stack([top, top / c["tau"] - (x / c["tau"]).logsumexp(1)], 1) *
                            torch.tensor([1.0, -1.0], device=DEV))
        p = torch.exp(lp)
        out["entropy"].append(-torch.where(p > 0.0, p * lp, 0.0).sum(1))
        out["logp"].append(torch.where(idx >= 0, lp.gather(1, idx.clamp(min=0)), 0.0))
        out["top_logp"].append(torch.sort(lp, 1, descending=True).values[:, :c["k"]])
    return {n: torch.cat(v) for n, v in out.items()} | {"top_idx": None}


def _exact_logp_grad(c, s):
    g = torch.zeros((c["N"], c["V"]), dtype=torch.float64, device=DEV)
    for r in range(0, c["N"], 256):
        rows = slice(r, r + 256)
        lp = torch.log_softmax(_f64(s["z"][rows]) / c["tau"], 1)
        p, idx = torch.exp(lp), s["idx"][rows]
        dl = s["d_logp"][rows].double() * (idx >= 0)
        g[rows].scatter_add_(1, idx.clamp(min=0), dl)
        g[rows] -= p * dl.sum(1, keepdim=True)
        if c["entropy"]:
            H = -(p * lp).sum(1, keepdim=True)
            g[rows] -= s["d_entropy"][rows].double()[:, None] * p * (lp + H)
    return {"g": _in(g * (s["grad_scale"] / c["tau"]), c["g"])}


def exact(case, seed):
    s = prepare(case, seed)
    return {"embed": _exact_embed, "embed_grad": _exact_embed_grad, "norm": _exact_norm,
            "norm_grad": _exact_norm_grad, "logp": _exact_logp,
            "logp_grad": _exact_logp_grad}[case["kind"]](case, s)


# ---- what a pass cannot do without ------------------------------------------------------------

def _distinct(T, V):
    """Different tokens among T, as expected."""
    r = torch.arange(1, V + 1, dtype=torch.float64)
    p = torch.log1p(1.0 / r) / math.log(V + 1.0) * (63.0 / 64.0)
    return int((1.0 - (1.0 - p) ** T).sum())


def work(case):
    c = case
    if c["kind"] == "embed":
        rows = _distinct(c["T"], c["V"])
        return {"bytes": 8 * c["T"] + c["W"] * (rows * _BYTES[c["table"]] + c["T"] * _BYTES[c["out"]]),
                "flops": c["T"] * c["W"]}
    if c["kind"] == "embed_grad":
        return {"bytes": 8 * c["T"] + c["W"] * (c["T"] * _BYTES[c["e"]] + c["V"] * _BYTES[c["g"]]),
                "flops": c["T"] * c["W"]}
    if c["kind"] == "norm":
        n = c["T"] * c["W"]
        return {"bytes": n * (_BYTES[c["x"]] + 2 * _BYTES[c["r"]] + _BYTES[c["y"]]) +
                c["W"] * _BYTES[c["w"]] + c["T"] * (8 if c["rows"] else 4), "flops": 6 * n}
    if c["kind"] == "norm_grad":
        n = c["T"] * c["W"]
        each = _BYTES[c["h"]] + _BYTES[c["dy"]] + _BYTES[c["d"]] * (2 if c["residual"] else 1) + 1
        return {"bytes": n * each + c["W"] * (_BYTES[c["w"]] + _BYTES[c["dw"]]) + 4 * c["T"],
                "flops": 10 * n}
    n = c["N"] * c["V"]
    if c["kind"] == "logp":
        return {"bytes": n * _BYTES[c["z"]] + c["N"] * (12 * c["m"] + 12 + 12 * c["k"]),
                "flops": 6 * n}
    return {"bytes": n * (_BYTES[c["z"]] + _BYTES[c["g"]]) +
            c["N"] * (12 * c["m"] + 12 + (4 if c["entropy"] else 0)), "flops": 6 * n}
