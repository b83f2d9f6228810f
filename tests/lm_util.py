"""Helpers of the language-model operators' GPU tests: random codes, last
roundings, and the comparison of a result's codes with a float64 value whose
error before the last rounding is bounded."""
import numpy as np
import torch

import oracle
import paper_1812_08011_amd as fp8t
from tests.gpu_util import DEV, dev, host

P8 = oracle.p8_value(np.arange(256, dtype=np.uint8))
P16 = oracle.p16_value(np.arange(65536, dtype=np.uint16))


def codes8(rng, shape, std=1.0):
    return oracle.fp8_quantize((rng.standard_normal(shape) * std).astype(np.float32))


def codes16(rng, shape, std=1.0):
    return oracle.fp16_quantize((rng.standard_normal(shape) * std).astype(np.float32))


def value(x):
    """float64 values of FP8 / FP16 codes or floats."""
    return P8[x] if x.dtype == np.uint8 else P16[x] if x.dtype == np.uint16 else x.astype(np.float64)


def step_error(x, dtype):
    """Half a step of the storage format at |x|: what the last rounding may add."""
    if dtype == np.float32:
        return np.abs(x) * 2.0 ** -24 + 2.0 ** -150
    bits, low = (3, 2.0 ** -17) if dtype == np.uint8 else (10, 2.0 ** -40)
    return np.maximum(np.abs(x) * 2.0 ** -bits, low)


def check(name, got, want, err):
    """got (codes or floats) within err, plus the last rounding, of want; NaN,
    Inf and finite values each where want has them."""
    val = value(got)
    ok_nan, fin = np.isnan(val) == np.isnan(want), np.isfinite(want)
    assert ok_nan.all(), (name, "NaN", np.argwhere(~ok_nan)[:5])
    inf = np.isinf(want)
    assert np.array_equal(val[inf], want[inf]), (name, "Inf")
    assert np.isfinite(val[fin]).all(), (name, "finite", np.argwhere(fin & ~np.isfinite(val))[:5])
    lim = err + step_error(np.abs(want) + err, got.dtype)
    with np.errstate(invalid="ignore"):
        bad = fin & (np.abs(val - want) > lim)
    assert not bad.any(), (name, int(bad.sum()), [(tuple(i), val[tuple(i)], want[tuple(i)],
                                                    lim[tuple(i)]) for i in np.argwhere(bad)[:5]])


def offsets(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)


def run_attention(q, k, v, cu_q, cu_k, causal, sm_scale, e=None, grad=np.uint16, scales=(1.0, 1.0),
                  strided=False, max_q=None, max_k=None, workspace=True):
    """attn_fwd_fp8 (and attn_bwd_fp8 with e) on host arrays; a dict of host
    results.  strided: operands and results as slices of wider buffers, the
    results' surroundings checked for stray writes."""
    torch_of = {np.uint16: torch.uint16, np.uint8: torch.uint8, np.float32: torch.float32}
    bufs = []

    def put(a):
        if not strided:
            return dev(a)
        T, H, D = a.shape
        wide = np.full((T, H + 1, D + 3), 0x7F, a.dtype)          # NaN around the operand
        wide[:, :H, 1:1 + D] = a
        return dev(wide)[:, :H, 1:1 + D]

    def out(shape, dtype):
        T, H, D = shape
        wide = torch.full((T, H + 1, D + 3) if strided else shape, 0x5A, dtype=torch.uint8,
                          device=DEV).to(torch.int32).to(torch_of[dtype])
        view = wide[:, :H, 1:1 + D] if strided else wide
        bufs.append((wide, shape, dtype))
        return view

    qd, kd, vd, ed = put(q), put(k), put(v), None if e is None else put(e)
    cq, ck = dev(np.asarray(cu_q, np.int64)), dev(np.asarray(cu_k, np.int64))
    nq, nk = np.diff(cu_q), np.diff(cu_k)
    args = (qd, kd, vd, cq, ck, int(nq.max(initial=0)) if max_q is None else max_q,
            int(nk.max(initial=0)) if max_k is None else max_k, causal, sm_scale)
    n = fp8t.attn_fwd_fp8_workspace_size(*args) if workspace else 0
    nb = fp8t.attn_bwd_fp8_workspace_size(*args)
    ws = torch.full((max(n, nb, 1),), 0xFF, dtype=torch.uint8, device=DEV)   # NaN to start with
    o, o8 = out(q.shape, np.uint16), out(q.shape, np.uint8)
    lse = torch.full((q.shape[1], q.shape[0]), np.nan, dtype=torch.float32, device=DEV)
    fp8t.attn_fwd_fp8(*args, o, o8, scales[0], lse, ws if n else None, n)
    res = dict(o=o, o8=o8, lse=lse)
    if e is not None:
        d = [out(q.shape, grad), out(k.shape, grad), out(v.shape, grad)]
        fp8t.attn_bwd_fp8(*args, o, ed, lse, *d, scales[1], ws, nb)
        res.update(zip(("dq", "dk", "dv"), d))
    got = {n: host(x) for n, x in res.items()}
    if strided:
        for wide, (T, H, D), dtype in bufs:
            w = host(wide).copy()
            w[:, :H, 1:1 + D] = 0x5A
            assert (w == 0x5A).all(), "a result was written outside its rows"
    return got
