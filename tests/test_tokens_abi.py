"""include/fp8train_tokens.h: every declared entry point is exported, and invalid
arguments are rejected before anything reaches the GPU (no compute call is made
here, so these run without one)."""
import os
import re

import pytest
import torch

import paper_1812_08011_amd as fp8t

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "fp8train_tokens.h")
FAKE = 0x10000        # never dereferenced: validation fails first
E = fp8t.EINVAL
BIG = 2 ** 31


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(fp8t.LIB_PATH):
        pytest.skip("libfp8train.so is not built")
    return fp8t.lib()


def test_declared_and_exported(lib):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"^\s*(?:int|size_t)\s+([a-z_0-9]+)\s*\(", text, flags=re.M)))
    assert names == ["embed_bwd", "embed_bwd_workspace_size", "embed_fwd", "rms_norm_bwd",
                     "rms_norm_bwd_workspace_size", "rms_norm_fwd", "token_logprobs",
                     "token_logprobs_bwd", "token_logprobs_workspace_size"]
    for name in names:
        assert hasattr(lib, name) and callable(getattr(fp8t, name)), name
    assert re.search(r"FP8T_MAX_TOP\s+%d\b" % fp8t.MAX_TOP, open(HEADER).read())
    assert fp8t.MAX_VOCAB == 1 << 24 and "FP8T_MAX_VOCAB (1 << 24)" in open(HEADER).read()
    assert fp8t.MAX_NORM_W == 1 << 20 and "FP8T_MAX_NORM_W (1 << 20)" in open(HEADER).read()


def caller(f, **defaults):
    def call(**kw):
        assert set(kw) <= set(defaults), kw
        return f(*{**defaults, **kw}.values(), None)
    return call


def test_embed_fwd_rejects(lib):
    call = caller(lib.embed_fwd, tok=FAKE, T=3, table=FAKE, tf=1, tld=8, V=5, W=8, scale=1.0, y=FAKE,
                  yf=2, yld=8)
    for bad in (dict(T=-1), dict(V=-1), dict(W=-1), dict(T=BIG), dict(V=BIG), dict(W=BIG, tld=BIG, yld=BIG),
                dict(tf=3), dict(tf=-1), dict(yf=3), dict(tld=7), dict(yld=7), dict(tok=None),
                dict(table=None), dict(y=None)):
        assert call(**bad) == E, bad
    assert call(T=0, tok=None, y=None) == fp8t.OK
    assert call(W=0) == fp8t.OK


def test_embed_bwd_rejects(lib):
    call = caller(lib.embed_bwd, tok=FAKE, T=3, e=FAKE, ef=1, eld=8, V=5, W=8, scale=1.0, g=FAKE, gf=1,
                  gld=8, ws=FAKE, wsb=1 << 20)
    for bad in (dict(T=-1), dict(V=-1), dict(W=-1), dict(T=BIG), dict(V=(1 << 24) + 1), dict(W=BIG, eld=BIG, gld=BIG),
                dict(ef=3), dict(gf=-1), dict(eld=7), dict(gld=0), dict(tok=None), dict(e=None),
                dict(g=None), dict(ws=FAKE + 8), dict(ws=None)):
        assert call(**bad) == E, bad
    need = lib.embed_bwd_workspace_size(3, 5, 8)
    assert need > 0 and call(wsb=need - 1) == call(ws=None, wsb=0) == fp8t.EWORKSPACE
    assert call(V=0, g=None) == call(W=0) == fp8t.OK
    assert lib.embed_bwd_workspace_size(-1, 5, 8) == lib.embed_bwd_workspace_size(3, 5, 0) == 0


def test_rms_norm_fwd_rejects(lib):
    call = caller(lib.rms_norm_fwd, x=FAKE, xf=1, xld=8, xs=None, r=FAKE, rld=8, w=FAKE, wf=1, T=3, W=8,
                  eps=1e-5, h=FAKE, sf=0, hld=8, y=FAKE, yf=2, yld=8, ys=1.0, yrs=None, rstd=FAKE)
    nan, inf = float("nan"), float("inf")
    for bad in (dict(T=-1), dict(W=-1), dict(T=BIG), dict(W=BIG, xld=BIG, rld=BIG, hld=BIG, yld=BIG),
                dict(W=2 ** 20 + 1, xld=BIG, rld=BIG, hld=BIG, yld=BIG),
                dict(xf=2), dict(sf=2), dict(wf=2), dict(yf=3), dict(xld=7), dict(rld=7), dict(hld=7),
                dict(yld=7), dict(x=None), dict(eps=0.0), dict(eps=-1e-5), dict(eps=nan), dict(eps=inf),
                dict(eps=1e-38), dict(h=None, y=None, rstd=None), dict(y=None, yrs=FAKE),
                dict(yrs=FAKE, ys=0.0), dict(yrs=FAKE, ys=-1.0), dict(yrs=FAKE, ys=inf),
                dict(yrs=FAKE, ys=nan)):
        assert call(**bad) == E, bad
    assert call(T=0, x=None) == call(W=0) == fp8t.OK


def test_rms_norm_bwd_rejects(lib):
    call = caller(lib.rms_norm_bwd, h=FAKE, hf=0, hld=8, w=FAKE, wf=1, rstd=FAKE, dy=FAKE, dyf=1, dyld=8,
                  dr=FAKE, drld=8, T=3, W=8, dx=FAKE, df=0, dxld=8, dx8=FAKE, dx8ld=8, s8=1.0, dw=FAKE,
                  dwf=0, ws=FAKE, wsb=1 << 20)
    for bad in (dict(T=-1), dict(W=-1), dict(T=BIG), dict(W=BIG, hld=BIG, dyld=BIG, drld=BIG, dxld=BIG, dx8ld=BIG),
                dict(W=2 ** 20 + 1, hld=BIG, dyld=BIG, drld=BIG, dxld=BIG, dx8ld=BIG),
                dict(hf=2), dict(wf=2), dict(dyf=3), dict(df=2), dict(dwf=2), dict(hld=7), dict(dyld=7),
                dict(drld=7), dict(dxld=7), dict(dx8ld=7), dict(h=None), dict(dy=None), dict(rstd=None),
                dict(dx=None, dx8=None, dw=None), dict(ws=FAKE + 4), dict(ws=None)):
        assert call(**bad) == E, bad
    need = lib.rms_norm_bwd_workspace_size(3, 8)
    assert need > 0 and call(wsb=need - 1) == call(ws=None, wsb=0) == fp8t.EWORKSPACE
    assert call(W=0) == fp8t.OK
    assert lib.rms_norm_bwd_workspace_size(0, 8) == lib.rms_norm_bwd_workspace_size(3, -8) == 0


LOGITS_BAD = (dict(N=-1), dict(V=-1), dict(V=0), dict(m=-1), dict(m=4097), dict(N=BIG), dict(V=BIG, zld=BIG),
              dict(V=2 ** 24 + 1, zld=BIG),
              dict(zf=2), dict(zld=49), dict(z=None), dict(tau=0.0), dict(tau=-1.0),
              dict(tau=float("nan")), dict(tau=float("inf")), dict(idx=None))


def test_token_logprobs_rejects(lib):
    call = caller(lib.token_logprobs, z=FAKE, zf=1, zld=50, idx=FAKE, m=2, N=3, V=50, tau=1.0, logp=FAKE,
                  entropy=FAKE, stats=FAKE, k=4, ti=FAKE, tl=FAKE, ws=None, wsb=0)
    for bad in LOGITS_BAD + (dict(k=-1), dict(k=129), dict(ws=None, wsb=64),
                             dict(logp=None, entropy=None, stats=None, ti=None, tl=None),
                             dict(logp=None, entropy=None, stats=None, k=0)):
        assert call(**bad) == E, bad
    assert call(N=0, z=None) == fp8t.OK
    big = dict(N=1, V=100000, zld=100000)
    need = lib.token_logprobs_workspace_size(1, 100000, 4)
    assert need > 0 and call(**big, ws=FAKE, wsb=need - 1) == fp8t.EWORKSPACE
    assert call(**big, ws=FAKE + 8, wsb=need) == E
    assert lib.token_logprobs_workspace_size(1, 100000, 129) == 0


def test_token_logprobs_bwd_rejects(lib):
    call = caller(lib.token_logprobs_bwd, z=FAKE, zf=1, zld=50, idx=FAKE, m=2, stats=FAKE, entropy=FAKE,
                  dl=FAKE, dh=FAKE, N=3, V=50, tau=1.0, s=1.0, g=FAKE, gf=1, gld=50)
    for bad in LOGITS_BAD + (dict(stats=None), dict(g=None), dict(gf=3), dict(gld=49),
                             dict(dl=None, dh=None), dict(entropy=None)):
        assert call(**bad) == E, bad
    assert call(N=0, z=None) == fp8t.OK


def test_binding_rejects():
    """What the binding refuses by itself: types, shapes, strides, devices."""
    f32 = lambda *s: torch.zeros(s)
    u16 = lambda *s: torch.zeros(s, dtype=torch.uint16)
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8)
    i64 = lambda *s: torch.zeros(s, dtype=torch.int64)
    def refused(error, f, *a, **kw):
        with pytest.raises(error):
            f(*a, **kw)
    refused(TypeError, fp8t.embed_fwd, i64(3), f32(5, 8).double(), f32(3, 8))
    refused(ValueError, fp8t.embed_fwd, i64(3), f32(5, 8), f32(3, 7))
    refused(ValueError, fp8t.embed_fwd, i64(3).int(), f32(5, 8), f32(3, 8))
    refused(ValueError, fp8t.embed_fwd, i64(3), f32(8, 5).T, f32(3, 8))
    refused(ValueError, fp8t.embed_bwd, i64(3), f32(4, 8), f32(5, 8))
    refused(ValueError, fp8t.embed_bwd, i64(3), f32(3, 8), f32(5, 8), 1.0, u8(16), 17)
    refused(TypeError, fp8t.rms_norm_fwd, u8(3, 8), None, None, 1e-5, None, u8(3, 8))
    refused(TypeError, fp8t.rms_norm_fwd, u16(3, 8), f32(3, 8), None, 1e-5, u16(3, 8), u8(3, 8))
    refused(ValueError, fp8t.rms_norm_fwd, u16(3, 8), None, u16(7), 1e-5, None, u8(3, 8))
    refused(ValueError, fp8t.rms_norm_fwd, u16(3, 8), None, None, 1e-5, None, u8(3, 8), rstd=f32(4))
    refused(TypeError, fp8t.rms_norm_bwd, f32(3, 8), None, f32(3), f32(3, 8), u16(3, 8), f32(3, 8))
    refused(ValueError, fp8t.rms_norm_bwd, f32(3, 8), None, f32(2), f32(3, 8), None, f32(3, 8))
    refused(TypeError, fp8t.token_logprobs, u8(2, 9), i64(2, 1), 1.0, f32(2, 1))
    refused(ValueError, fp8t.token_logprobs, f32(2, 9), i64(2, 1), 1.0, f32(2, 2))
    refused(ValueError, fp8t.token_logprobs, f32(2, 9), None, 1.0, top_idx=i64(2, 3), top_logp=f32(2, 4))
    refused(ValueError, fp8t.token_logprobs_bwd, f32(2, 9), i64(2, 1), 1.0, f32(2, 2), None, f32(2, 2),
            None, 1.0, f32(2, 9))
    # well-formed calls on tensors that are not on the GPU
    refused(ValueError, fp8t.embed_fwd, i64(3), f32(5, 8), f32(3, 8))
    refused(ValueError, fp8t.embed_bwd, i64(3), f32(3, 8), f32(5, 8))
    refused(ValueError, fp8t.rms_norm_fwd, f32(3, 8), None, None, 1e-5, None, u8(3, 8))
    refused(ValueError, fp8t.rms_norm_bwd, f32(3, 8), None, f32(3), f32(3, 8), None, f32(3, 8))
    refused(ValueError, fp8t.token_logprobs, f32(2, 9), i64(2, 1), 1.0, f32(2, 1))
    refused(ValueError, fp8t.token_logprobs_bwd, f32(2, 9), i64(2, 1), 1.0, f32(2, 2), None, f32(2, 1),
            None, 1.0, f32(2, 9))
