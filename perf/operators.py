"""Measured cases of the language-model operators around the FP8 GEMMs.

Three operators of one training step of a language model in the paper's
formats: rotary positions, attention over packed sequences (forward and
backward), and the distillation loss from a teacher's top logits with its
gradient.  ``run`` makes one pass: with ``own`` true through the package's
public functions, with ``own`` false in elementary torch operations in 32 bits,
rounded once at the end.

Formats: FP8 (1,5,2) codes in uint8 are torch's float8_e5m2 bit for bit and
come back as that type.  FP16 (1,6,9) codes in uint16 have no torch type; a
result in FP16 comes back as IEEE half, which holds every FP16 value from 2^-14
to 2^16 exactly (fp16_dequantize).

Kinds:

* ``rotary``  -- rotation of the query and key heads of a projection's result.
* ``attn``    -- ``train`` false: attention forward (result in FP8 and the rows'
  log-sum-exp); true: forward and backward, with the three gradients.
* ``distill`` -- per-row loss and the gradient of the logits.
"""
import math

import torch

own = False
DEV = "cuda:0"


def listed():
    return [
        # one token of one sequence: what a step of generation rotates
        dict(name="rotary_token", kind="rotary", T=1, H=10, D=64, R=64, layout="half", inverse=False,
             out="fp8", base=10000.0, mscale=1.0, first=5000, seq=1),
        # query and key heads of a long packed batch, scaled for long contexts
        dict(name="rotary_prompt", kind="rotary", T=16384, H=40, D=128, R=128, layout="half",
             inverse=False, out="fp8", base=500000.0, mscale=1.2, first=0, seq=16384),
        # gradient of a rotation of part of the head: odd token count, interleaved pairs
        dict(name="rotary_part_backward", kind="rotary", T=5003, H=12, D=80, R=48,
             layout="interleaved", inverse=True, out="fp16", base=10000.0, mscale=1.0, first=7,
             seq=1001),
        # eight sequences each asking with one token over their own history
        dict(name="attn_token", kind="attn", train=False, lens_q="1,1,1,1,1,1,1,1",
             lens_k="8192,1,777,4096,33,6001,2500,129", Hq=32, Hkv=8, D=128, causal=True, grad=""),
        # many short sequences in one batch
        dict(name="attn_short", kind="attn", train=False,
             lens_q="5,96,33,64,1,17,80,41,2,90,65,7,31,32,55,12,3,77,48,66,29,94,10,61", lens_k="",
             Hq=16, Hkv=16, D=64, causal=True, grad=""),
        # one long prompt with grouped heads
        dict(name="attn_prompt", kind="attn", train=False, lens_q="16384", lens_k="", Hq=8, Hkv=2,
             D=128, causal=True, grad=""),
        # a packed training batch of mixed lengths, gradients in FP8 for the next GEMMs
        dict(name="attn_train_packed", kind="attn", train=True, lens_q="1,17,700,1024,333,2021,4096",
             lens_k="", Hq=16, Hkv=16, D=64, causal=True, grad="fp8"),
        # a long training sequence with grouped heads, gradients in FP16
        dict(name="attn_train_long", kind="attn", train=True, lens_q="8192", lens_k="", Hq=16, Hkv=4,
             D=128, causal=True, grad="fp16"),
        # an encoder's batch: no causal mask, sizes that fit no tile
        dict(name="attn_train_odd", kind="attn", train=True, lens_q="257,1000,63,129", lens_k="",
             Hq=6, Hkv=3, D=80, causal=False, grad="fp16"),
        # the framework's own last layer (6000 outputs, batch 256) with its FP16 error
        dict(name="distill_last_layer", kind="distill", N=256, V=6000, k=8, tau=2.0, z="fp16",
             out="fp16", padded=False),
        # a language model's logits, the error in FP8 for the GEMMs that follow
        dict(name="distill_vocab", kind="distill", N=4096, V=32768, k=64, tau=1.0, z="fp16",
             out="fp8", padded=True),
        # FP32 logits, odd sizes, rows without a target
        dict(name="distill_f32", kind="distill", N=777, V=50001, k=20, tau=4.0, z="f32", out="f32",
             padded=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_rotary(rng):
    D = rng.choice([32, 64, 80, 96, 128, 128, 100])
    part = rng.random() < 0.3
    R = max(2, int(D * rng.choice([0.25, 0.5, 0.6])) // 2 * 2) if part else D
    H = rng.randint(1, 40)
    T = _log_int(rng, 1, max(1, 16384 * 40 * 128 // (H * D)))
    return dict(kind="rotary", T=T, H=H, D=D, R=R, layout=rng.choice(["half", "interleaved"]),
                inverse=rng.random() < 0.4, out=rng.choice(["fp8", "fp8", "fp16"]),
                base=rng.choice([10000.0, 500000.0]), mscale=rng.choice([1.0, 1.0, 1.2]),
                first=_log_int(rng, 1, 60000), seq=_log_int(rng, 1, 65536))


def _draw_attn(rng):
    train = rng.random() < 0.5
    D = rng.choice([32, 64, 64, 80, 96, 128, 128, 40])
    Hkv = rng.choice([1, 2, 3, 4, 8])
    Hq = Hkv * rng.choice([1, 1, 2, 3, 4, 8])
    cap = (400e6 if train else 800e6) / Hq
    if not train and rng.random() < 0.4:            # few new tokens over a long history
        n = rng.randint(1, 16)
        lk = [_log_int(rng, 1, 16384) for _ in range(n)]
        lq = [min(m, rng.choice([1, 1, 1, 2, 5])) for m in lk]
        while sum(lq) * sum(lk) > cap:
            lk = [max(1, m // 2) for m in lk]
            lq = [min(a, b) for a, b in zip(lq, lk)]
        return dict(kind="attn", train=False, lens_q=",".join(map(str, lq)),
                    lens_k=",".join(map(str, lk)), Hq=Hq, Hkv=Hkv, D=D, causal=True, grad="")
    n, total = rng.randint(1, 12), _log_int(rng, 64, int(min(12000, math.sqrt(cap))))
    cuts = sorted(rng.randint(0, total) for _ in range(n - 1))
    lens = [b - a for a, b in zip([0] + cuts, cuts + [total]) if b > a]
    return dict(kind="attn", train=train, lens_q=",".join(map(str, lens)), lens_k="", Hq=Hq, Hkv=Hkv,
                D=D, causal=rng.random() < 0.75, grad=rng.choice(["fp8", "fp16"]) if train else "")


def _draw_distill(rng):
    V = _log_int(rng, 500, 131072)
    N = _log_int(rng, 1, max(1, min(8192, 4096 * 32768 // (2 * V))))
    z = rng.choice(["fp16", "fp16", "f32"])
    return dict(kind="distill", N=N, V=V, k=rng.choice([1, 5, 16, 50, 64, 100]),
                tau=rng.choice([1.0, 2.0, 4.0]), z=z,
                out=rng.choice(["fp16", "fp8"]) if z == "fp16" else "f32",
                padded=rng.random() < 0.5 and N > 4)


def draw(rng):
    kind = rng.choice(["rotary", "attn", "attn", "attn", "distill", "distill"])
    return {"rotary": _draw_rotary, "attn": _draw_attn, "distill": _draw_distill}[kind](rng)


# ---- the storage formats in torch operations ----------------------------------------

def _round16(x):
    """float32 -> nearest FP16 (1,6,9) value, ties to even, as float32."""
    u = x.view(torch.int32)
    r = ((u + 0x1FFF + ((u >> 14) & 1)) & ~0x3FFF).view(torch.float32)
    low = torch.round(x * 2.0 ** 39) * 2.0 ** -39          # below 2^-30 the step is 2^-39
    return torch.where(x.abs() < 2.0 ** -30, low, r)


def _encode16(x):
    """float32 -> FP16 codes (uint16), for finite values below 2^32."""
    r = _round16(x)
    u = r.view(torch.int32) & 0x7FFFFFFF
    code = torch.where(r.abs() < 2.0 ** -30, (r.abs() * 2.0 ** 39).to(torch.int32),
                       (u >> 14) - (96 << 9))
    code = code | torch.where(r < 0, 0x8000, 0).to(torch.int32)
    return code.to(torch.int16).view(torch.uint16)


def _decode16(c):
    """FP16 codes of finite values -> float32: exponent and significand moved into
    float32's fields, the exponents' bias (127 - 31) restored by a product."""
    i = c.view(torch.int16).to(torch.int32)
    return ((i << 14) & -1610612737).view(torch.float32) * 2.0 ** 96


def _decode8(c):
    return c.view(torch.float8_e5m2).to(torch.float32)


def _encode8(x):
    return x.clamp(-57344.0, 57344.0).to(torch.float8_e5m2)


def _as(x, out):
    """float32 results in the storage type `out`, as the values that come back."""
    return x if out == "f32" else _encode8(x) if out == "fp8" else _round16(x).to(torch.float16)


_BYTES = {"f32": 4, "fp16": 2, "fp8": 1}
_DTYPE = {"f32": torch.float32, "fp16": torch.uint16, "fp8": torch.uint8}


def _buffer(out, *shape):
    return torch.empty(shape, dtype=_DTYPE[out], device=DEV)


def _values(buf, out, half):
    """An operator's result as values: FP16 codes through the package's decoder."""
    if out != "fp16":
        return buf.view(torch.float8_e5m2) if out == "fp8" else buf
    import paper_1812_08011_amd as fp8t
    return fp8t.fp16_dequantize(buf, half)


# ---- inputs ---------------------------------------------------------------------------

def _normal(gen, shape, std=1.0):
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32) * std


def _lens(c):
    q = [int(x) for x in c["lens_q"].split(",")]
    return q, [int(x) for x in c["lens_k"].split(",")] if c["lens_k"] else q


def _offsets(lens):
    return torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int64, device=DEV)


def _prepare_rotary(c, gen):
    T, H, D, R = c["T"], c["H"], c["D"], c["R"]
    s = dict(c)
    s["x"] = _encode16(_normal(gen, (T, H, D)))
    s["positions"] = c["first"] + torch.arange(T, device=DEV) % c["seq"]
    # by-parts scaling for contexts eight times longer: slow pairs slowed down
    freqs = c["base"] ** (-torch.arange(0, R, 2, dtype=torch.float64, device=DEV) / R)
    if c["mscale"] != 1.0:
        turns = freqs * 4096.0 / (2.0 * math.pi)
        keep = ((turns - 1.0) / 31.0).clamp(0.0, 1.0)
        freqs = freqs * keep + freqs / 8.0 * (1.0 - keep)
    s["freqs"] = freqs
    s["y"] = _buffer(c["out"], T, H, D)
    s["half"] = torch.empty((T, H, D), dtype=torch.float16, device=DEV)
    return s


def _prepare_attn(c, gen):
    lq, lk = _lens(c)
    Tq, Tk, Hq, Hkv, D = sum(lq), sum(lk), c["Hq"], c["Hkv"], c["D"]
    s = dict(c, Tq=Tq, Tk=Tk, max_q=max(lq), max_k=max(lk), sm_scale=1.0 / math.sqrt(D), ws={})
    # one projection's result: queries and keys from one buffer where their counts agree
    codes = lambda T, H: _encode8(_normal(gen, (T, H, D))).view(torch.uint8)
    if Tq == Tk:
        qkv = codes(Tq, Hq + 2 * Hkv)
        s["q"], s["k"], s["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    else:
        s["q"], s["k"], s["v"] = codes(Tq, Hq), codes(Tk, Hkv), codes(Tk, Hkv)
    s["cu_q"], s["cu_k"] = _offsets(lq), _offsets(lk)
    s["o8"], s["lse"] = _buffer("fp8", Tq, Hq, D), _buffer("f32", Hq, Tq)
    if c["train"]:
        # the error of the output projection under a loss scale of 1024
        s["do"] = _encode8(_normal(gen, (Tq, Hq, D), 1e-3) * 1024.0).view(torch.uint8)
        s["o16"] = _buffer("fp16", Tq, Hq, D)
        for n, T, H in (("dq", Tq, Hq), ("dk", Tk, Hkv), ("dv", Tk, Hkv)):
            s[n] = _buffer(c["grad"], T, H, D)
            s[n + "_half"] = torch.empty((T, H, D), dtype=torch.float16, device=DEV)
    return s


def _prepare_distill(c, gen):
    N, V, k = c["N"], c["V"], c["k"]
    s = dict(c)
    z = _normal(gen, (N, V), 2.0)
    # k distinct entries of each row, on which the student partly agrees
    first = torch.randint(0, V, (N, 1), generator=gen, device=DEV)
    idx = (first + torch.arange(k, device=DEV) * (V // k)) % V
    t = torch.sort(_normal(gen, (N, k), 2.0), dim=1, descending=True).values + 6.0
    z.scatter_add_(1, idx, t * 0.7)
    w = torch.full((N,), 1.0 / N, device=DEV)
    if c["padded"]:
        # some rows are padding, and the teacher gave fewer entries for some rows
        w = torch.where(torch.rand((N,), generator=gen, device=DEV) < 0.1, 0.0, w)
        few = torch.randint(1, k + 1, (N, 1), generator=gen, device=DEV)
        idx = torch.where(torch.arange(k, device=DEV) < few, idx, -1)
    s["z"] = _encode16(z) if c["z"] == "fp16" else z
    s["idx"], s["t"], s["w"] = idx.contiguous(), t, w
    s["grad_scale"] = 1024.0 * N
    s["loss"], s["g"] = _buffer("f32", N), _buffer(c["out"], N, V)
    if c["out"] == "fp16":
        s["half"] = torch.empty((N, V), dtype=torch.float16, device=DEV)
    return s


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return {"rotary": _prepare_rotary, "attn": _prepare_attn,
            "distill": _prepare_distill}[case["kind"]](case, gen)


# ---- one pass through the framework -----------------------------------------------------

def _own_rotary(s):
    import paper_1812_08011_amd as fp8t
    fp8t.rotary_embed(s["x"], s["positions"], s["freqs"], s["y"], s["layout"] == "interleaved",
                      s["inverse"], s["mscale"], 1.0)
    return {"y": _values(s["y"], s["out"], s["half"])}


def _own_attn(s):
    import paper_1812_08011_amd as fp8t
    args = (s["q"], s["k"], s["v"], s["cu_q"], s["cu_k"], s["max_q"], s["max_k"], s["causal"],
            s["sm_scale"])
    if "bytes" not in s["ws"]:                              # a program keeps its workspace
        n = fp8t.attn_fwd_fp8_workspace_size(*args)
        if s["train"]:
            n = max(n, fp8t.attn_bwd_fp8_workspace_size(*args))
        s["ws"]["bytes"] = n
        s["ws"]["buffer"] = torch.empty(n, dtype=torch.uint8, device=DEV) if n else None
    ws = (s["ws"]["buffer"], s["ws"]["bytes"])
    fp8t.attn_fwd_fp8(*args, s.get("o16"), s["o8"], 1.0, s["lse"], *ws)
    out = {"o": s["o8"].view(torch.float8_e5m2), "lse": s["lse"]}
    if s["train"]:
        fp8t.attn_bwd_fp8(*args, s["o16"], s["do"], s["lse"], s["dq"], s["dk"], s["dv"], 1.0, *ws)
        out.update({n: _values(s[n], s["grad"], s[n + "_half"]) for n in ("dq", "dk", "dv")})
    return out


def _own_distill(s):
    import paper_1812_08011_amd as fp8t
    fp8t.distill_loss(s["z"], s["idx"], s["t"], s["w"], s["tau"], s["grad_scale"], s["loss"], s["g"])
    return {"loss": s["loss"], "g": _values(s["g"], s["out"], s.get("half"))}


# ---- the same in elementary torch operations ----------------------------------------------

def _plain_rotary(s):
    x, R = _decode16(s["x"]), s["R"]
    angle = s["positions"].to(torch.float32)[:, None] * s["freqs"].to(torch.float32)
    cos, sin = torch.cos(angle)[:, None] * s["mscale"], torch.sin(angle)[:, None] * s["mscale"]
    sin = -sin if s["inverse"] else sin
    if s["layout"] == "half":
        a, b = x[..., :R // 2], x[..., R // 2:R]
        rotated = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = x[..., 0:R:2], x[..., 1:R:2]
        rotated = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return {"y": _as(torch.cat([rotated, x[..., R:]], -1), s["out"])}


def _visible(s):
    """Tq x Tk: whether a query sees a key (same sequence; causal: aligned to its end)."""
    iq, ik = torch.arange(s["Tq"], device=DEV), torch.arange(s["Tk"], device=DEV)
    sq = torch.searchsorted(s["cu_q"], iq, right=True) - 1
    sk = torch.searchsorted(s["cu_k"], ik, right=True) - 1
    see = sq[:, None] == sk
    if s["causal"]:
        # distance of the query and of the key from the end of their sequence
        see &= (s["cu_k"][1:][sk] - ik) >= (s["cu_q"][1:][sq] - iq)[:, None]
    return see


def _plain_attn(s):
    Hq, Hkv, D, Tq, Tk, c = s["Hq"], s["Hkv"], s["D"], s["Tq"], s["Tk"], s["sm_scale"]
    G = Hq // Hkv
    heads_q = lambda x: _decode8(x).reshape(Tq, Hkv, G, D).permute(1, 2, 0, 3).reshape(Hkv, -1, D)
    heads_k = lambda x: _decode8(x).permute(1, 0, 2).contiguous()
    tokens_q = lambda x: x.reshape(Hkv, G, Tq, D).permute(2, 0, 1, 3).reshape(Tq, Hq, D)
    tokens_k = lambda x: x.permute(1, 0, 2)
    q, k, v = heads_q(s["q"]), heads_k(s["k"]), heads_k(s["v"])
    see = _visible(s)
    S = (torch.matmul(q, k.transpose(1, 2)) * c).view(Hkv, G, Tq, Tk)
    S = S.masked_fill_(~see, -math.inf)
    m = S.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)                 # a row that sees nothing
    P = torch.exp(S.sub_(m))
    l = P.sum(-1, keepdim=True)
    P = P.div_(torch.where(l == 0.0, 1.0, l)).view(Hkv, G * Tq, Tk)
    o = torch.matmul(P, v)
    out = {"o": _as(tokens_q(o).contiguous(), "fp8"), "lse": (torch.log(l) + m).reshape(Hq, Tq)}
    if s["train"]:
        do = heads_q(s["do"])
        dP = torch.matmul(do, v.transpose(1, 2))
        delta = (do * o).sum(-1, keepdim=True)
        dS = dP.sub_(delta).mul_(P).mul_(c)
        g = s["grad"]
        out["dq"] = _as(tokens_q(torch.matmul(dS, k)).contiguous(), g)
        out["dk"] = _as(tokens_k(torch.matmul(dS.transpose(1, 2), q)).contiguous(), g)
        out["dv"] = _as(tokens_k(torch.matmul(P.transpose(1, 2), do)).contiguous(), g)
    return out


def _plain_distill(s):
    z = (_decode16(s["z"]) if s["z"].dtype == torch.uint16 else s["z"]) / s["tau"]
    used = s["idx"] >= 0
    t = (s["t"] / s["tau"]).masked_fill(~used, -math.inf)
    q = torch.exp(t - t.amax(1, keepdim=True))
    q = q / q.sum(1, keepdim=True)
    m = z.amax(1, keepdim=True)
    e = torch.exp(z - m)
    l = e.sum(1, keepdim=True)
    at = s["idx"].clamp(min=0)
    logp = torch.gather(z, 1, at) - m - torch.log(l)
    kl = torch.where(used, q * (torch.log(torch.where(used, q, 1.0)) - logp), 0.0).sum(1)
    g = (e / l).scatter_add(1, at, torch.where(used, -q, 0.0))
    w = s["w"]
    return {"loss": w * s["tau"] ** 2 * kl,
            "g": _as(g * (w * (s["tau"] * s["grad_scale"]))[:, None], s["out"])}


def run(state):
    if own:
        return {"rotary": _own_rotary, "attn": _own_attn, "distill": _own_distill}[state["kind"]](state)
    return {"rotary": _plain_rotary, "attn": _plain_attn,
            "distill": _plain_distill}[state["kind"]](state)


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
    return torch.where((i >> (eb + mb)) & 1 == 1, -mag, mag)


def _exact_rotary(c, s):
    x, R = _f64(s["x"]), c["R"]
    z = s["positions"].double()[:, None] * s["freqs"]
    turn = torch.polar(torch.full_like(z, c["mscale"]), -z if c["inverse"] else z)[:, None]
    n = R // 2
    first = torch.arange(n, device=DEV) * (1 if c["layout"] == "half" else 2)
    second = first + (n if c["layout"] == "half" else 1)
    pairs = torch.complex(x[..., first], x[..., second]) * turn
    y = x.clone()
    y[..., first], y[..., second] = pairs.real, pairs.imag
    return {"y": y}


def _exact_attn(c, s):
    lq, lk = _lens(c)
    G, D = c["Hq"] // c["Hkv"], c["D"]
    q, k, v = _f64(s["q"]), _f64(s["k"]), _f64(s["v"])
    o, lse = torch.zeros_like(q), torch.full((c["Hq"], q.shape[0]), -math.inf, dtype=q.dtype, device=DEV)
    out = {"o": o, "lse": lse}
    if c["train"]:
        do = _f64(s["do"])
        out.update(dq=torch.zeros_like(q), dk=torch.zeros_like(k), dv=torch.zeros_like(v))
    a = b = 0
    for nq, nk in zip(lq, lk):
        for h in range(c["Hq"]):
            Q, K, V = q[a:a + nq, h], k[b:b + nk, h // G], v[b:b + nk, h // G]
            S = Q @ K.T / math.sqrt(D)
            if c["causal"]:
                S += torch.full((nq, nk), -math.inf, dtype=S.dtype, device=DEV).triu(nk - nq + 1)
            L = torch.logsumexp(S, 1)
            P = torch.exp(S - L[:, None])
            lse[h, a:a + nq] = L
            o[a:a + nq, h] = P @ V
            if c["train"]:
                E = do[a:a + nq, h]
                dP = E @ V.T
                dS = P * (dP - (P * dP).sum(1, keepdim=True)) / math.sqrt(D)
                out["dq"][a:a + nq, h] = dS @ K
                out["dk"][b:b + nk, h // G] += dS.T @ Q
                out["dv"][b:b + nk, h // G] += P.T @ E
        a, b = a + nq, b + nk
    return out


def _exact_distill(c, s):
    tau, N = c["tau"], c["N"]
    loss = torch.zeros(N, dtype=torch.float64, device=DEV)
    g = torch.zeros(N, c["V"], dtype=torch.float64, device=DEV)
    step = max(1, 2 ** 26 // c["V"])
    for r in range(0, N, step):
        rows = slice(r, min(N, r + step))
        idx, used = s["idx"][rows], s["idx"][rows] >= 0
        logq = torch.log_softmax(torch.where(used, s["t"][rows].double() / tau, -math.inf), 1)
        logp = torch.log_softmax(_f64(s["z"][rows]) / tau, 1)
        q = torch.exp(logq)
        terms = q * (logq - logp.gather(1, idx.clamp(min=0)))
        w = s["w"][rows].double()
        loss[rows] = w * tau ** 2 * torch.where(used, terms, 0.0).sum(1)
        d = torch.exp(logp)
        d.scatter_add_(1, idx.clamp(min=0), -q)
        g[rows] = d * (w * tau * s["grad_scale"])[:, None]
    return {"loss": loss, "g": g}


def exact(case, seed):
    s = prepare(case, seed)
    return {"rotary": _exact_rotary, "attn": _exact_attn, "distill": _exact_distill}[case["kind"]](case, s)


# ---- what a pass cannot do without ------------------------------------------------------------

def _pairs(c):
    """(query, key) pairs of one head that the mask leaves."""
    lq, lk = _lens(c)
    if not c["causal"]:
        return sum(a * b for a, b in zip(lq, lk))
    # query i of a sequence sees its first i + 1 + nk - nq keys
    seen = lambda a, b: a * (b - a) + a * (a + 1) // 2 if b >= a else b * (b + 1) // 2
    return sum(seen(a, b) for a, b in zip(lq, lk))


def work(case):
    c = case
    if c["kind"] == "rotary":
        n = c["T"] * c["H"] * c["D"]
        return {"bytes": n * (2 + _BYTES[c["out"]]) + 8 * c["T"] + 4 * c["R"],
                "flops": 3 * c["T"] * c["H"] * c["R"]}
    if c["kind"] == "attn":
        lq, lk = _lens(c)
        rows, keys, D = sum(lq) * c["Hq"], sum(lk) * c["Hkv"], c["D"]
        nbytes, flops = 2 * rows * D + 4 * rows + 2 * keys * D, 4 * D * c["Hq"] * _pairs(c)
        if c["train"]:
            # the error read; dq, dk and dv written; five more products than the forward's two
            nbytes += rows * D + _BYTES[c["grad"]] * D * (rows + 2 * keys)
            flops += 10 * D * c["Hq"] * _pairs(c)
        return {"bytes": nbytes, "flops": flops}
    N, V = c["N"], c["V"]
    return {"bytes": N * V * (_BYTES[c["z"]] + _BYTES[c["out"]]) + N * (12 * c["k"] + 8),
            "flops": 6 * N * V}
