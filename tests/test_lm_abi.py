"""include/fp8train_lm.h: every declared entry point is exported, and invalid
arguments are rejected before anything reaches the GPU (no compute call is
made here, so these run without one)."""
import os
import re

import pytest

import paper_1812_08011_amd as fp8t

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "fp8train_lm.h")
FAKE = 0x10000        # never dereferenced: validation fails first
E = fp8t.EINVAL


def declared_functions():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    return sorted(set(re.findall(r"^\s*(?:int|size_t)\s+([a-z_0-9]+)\s*\(", text, flags=re.M)))


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(fp8t.LIB_PATH):
        pytest.skip("libfp8train.so is not built")
    return fp8t.lib()


def test_declared_and_exported(lib):
    assert declared_functions() == [
        "attn_bwd_fp8", "attn_bwd_fp8_workspace_size", "attn_fwd_fp8",
        "attn_fwd_fp8_workspace_size", "distill_loss", "fp16_dequantize", "rotary_embed"]
    for name in declared_functions():
        assert hasattr(lib, name) and callable(getattr(fp8t, name)), name


def test_dequantize_rejects(lib):
    f = lib.fp16_dequantize
    assert f(FAKE, 1.0, FAKE, fp8t.FMT_F32, -1, None) == E
    assert f(FAKE, 1.0, FAKE, fp8t.FMT_FP8, 4, None) == E
    assert f(None, 1.0, FAKE, fp8t.FMT_HALF, 4, None) == E
    assert f(FAKE, 1.0, None, fp8t.FMT_HALF, 4, None) == E
    assert f(None, 1.0, None, fp8t.FMT_F32, 0, None) == fp8t.OK


def test_rotary_rejects(lib):
    def call(**kw):
        a = dict(x=FAKE, xf=1, xts=128, xhs=64, pos=FAKE, fr=FAKE, T=3, H=2, D=64, R=64, il=0, inv=0,
                 m=1.0, s=1.0, y=FAKE, yf=2, yts=128, yhs=64)
        a.update(kw)
        return lib.rotary_embed(a["x"], a["xf"], a["xts"], a["xhs"], a["pos"], a["fr"], a["T"], a["H"],
                                a["D"], a["R"], a["il"], a["inv"], a["m"], a["s"], a["y"], a["yf"],
                                a["yts"], a["yhs"], None)
    for bad in (dict(T=-1), dict(H=-1), dict(D=-1), dict(R=65), dict(R=3), dict(R=-2), dict(xf=3),
                dict(yf=-1), dict(il=2), dict(inv=-1), dict(xts=-1), dict(xhs=-64), dict(yhs=63),
                dict(yts=127), dict(yts=0), dict(x=None), dict(y=None), dict(pos=None), dict(fr=None),
                dict(D=65537, R=0, yts=1 << 20, yhs=1 << 18), dict(T=2 ** 31)):
        assert call(**bad) == E, bad
    assert call(T=0) == fp8t.OK
    assert call(H=0, x=None) == fp8t.OK


def attn_args(bwd, **kw):
    a = dict(q=FAKE, qts=128, qhs=64, k=FAKE, kts=64, khs=64, v=FAKE, vts=64, vhs=64, cq=FAKE, ck=FAKE,
             S=1, Tq=4, Tk=4, mq=4, mk=4, Hq=2, Hkv=1, D=64, causal=1, c=0.125, o=FAKE, ots=128, ohs=64,
             o8=FAKE, o8ts=128, o8hs=64, o8s=1.0, lse=FAKE, e=FAKE, ets=128, ehs=64, dq=FAKE, dqts=128,
             dqhs=64, dk=FAKE, dkts=64, dkhs=64, dv=FAKE, dvts=64, dvhs=64, gf=1, gs=1.0, ws=None, wsb=0)
    a.update(kw)
    common = ["q", "qts", "qhs", "k", "kts", "khs", "v", "vts", "vhs", "cq", "ck", "S", "Tq", "Tk", "mq",
              "mk", "Hq", "Hkv", "D", "causal", "c", "o", "ots", "ohs"]
    rest = ["e", "ets", "ehs", "lse", "dq", "dqts", "dqhs", "dk", "dkts", "dkhs", "dv", "dvts", "dvhs",
            "gf", "gs"] if bwd else ["o8", "o8ts", "o8hs", "o8s", "lse"]
    return [a[n] for n in common + rest + ["ws", "wsb"]] + [None]


SHARED_BAD = [dict(S=-1), dict(Tq=-1), dict(Tk=-1), dict(mq=-1), dict(mk=-2), dict(Hq=3, Hkv=2),
              dict(Hkv=0), dict(Hq=-2), dict(D=0), dict(D=129), dict(causal=2), dict(causal=-1),
              dict(c=0.0), dict(c=-1.0), dict(c=float("nan")), dict(c=float("inf")), dict(qts=-1),
              dict(khs=-1), dict(vts=-5), dict(q=None), dict(k=None), dict(v=None), dict(cq=None),
              dict(ck=None), dict(Tq=2 ** 31), dict(Tk=2 ** 31), dict(ws=None, wsb=64)]


def test_attn_fwd_rejects(lib):
    call = lambda **kw: lib.attn_fwd_fp8(*attn_args(False, **kw))
    for bad in SHARED_BAD + [dict(ohs=63), dict(ots=127), dict(o8ts=100), dict(o8hs=0),
                             dict(o=None, o8=None, lse=None)]:
        assert call(**bad) == E, bad
    assert call(Tq=0) == fp8t.OK
    assert call(S=0) == fp8t.OK
    assert call(Hq=0, Hkv=0) == fp8t.OK
    assert fp8t.lib().attn_fwd_fp8_workspace_size(1, 4, 4, 4, 4, 2, 1, 200, 1) == 0


def test_attn_bwd_rejects(lib):
    call = lambda **kw: lib.attn_bwd_fp8(*attn_args(True, **{**dict(ws=FAKE, wsb=1 << 20), **kw}))
    for bad in SHARED_BAD + [dict(e=None), dict(o=None), dict(lse=None), dict(dq=None), dict(dk=None),
                             dict(dv=None), dict(gf=0), dict(gf=3), dict(dqhs=10), dict(dkts=63),
                             dict(dvts=0), dict(ets=-1), dict(ws=FAKE + 4)]:
        assert call(**bad) == E, bad
    assert call(ws=None, wsb=0) == fp8t.EWORKSPACE
    need = lib.attn_bwd_fp8_workspace_size(1, 4, 4, 4, 4, 2, 1, 64, 1)
    assert need > 0 and call(wsb=need - 1) == fp8t.EWORKSPACE
    assert call(S=0) == fp8t.OK


def test_distill_rejects(lib):
    def call(**kw):
        a = dict(z=FAKE, zf=1, zld=50, idx=FAKE, t=FAKE, tf=0, k=4, w=None, N=3, V=50, tau=1.0, s=1.0,
                 loss=FAKE, g=FAKE, gf=1, gld=50)
        a.update(kw)
        return lib.distill_loss(a["z"], a["zf"], a["zld"], a["idx"], a["t"], a["tf"], a["k"], a["w"],
                                a["N"], a["V"], a["tau"], a["s"], a["loss"], a["g"], a["gf"], a["gld"],
                                None)
    for bad in (dict(N=-1), dict(V=-1), dict(k=-1), dict(k=4097), dict(zf=2), dict(tf=2), dict(gf=3),
                dict(gf=-1), dict(tau=0.0), dict(tau=-1.0), dict(tau=float("nan")),
                dict(tau=float("inf")), dict(zld=49), dict(gld=49), dict(z=None), dict(idx=None),
                dict(t=None), dict(loss=None, g=None), dict(V=2 ** 31, zld=2 ** 32, gld=2 ** 32),
                dict(N=2 ** 31)):
        assert call(**bad) == E, bad
    assert call(N=0) == fp8t.OK


def test_binding_rejects():
    """What the binding refuses by itself: types, shapes, strides."""
    import torch
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8)
    i64 = lambda *s: torch.zeros(s, dtype=torch.int64)
    q, k, cu = u8(4, 2, 8), u8(4, 1, 8), i64(2)
    with pytest.raises(TypeError):
        fp8t.attn_fwd_fp8(q.float(), k, k, cu, cu, 4, 4, True, 1.0, None, q)
    with pytest.raises(ValueError):
        fp8t.attn_fwd_fp8(q, k, u8(5, 1, 8), cu, cu, 4, 4, True, 1.0, None, q)
    with pytest.raises(ValueError):
        fp8t.attn_fwd_fp8(q, u8(4, 1, 7), u8(4, 1, 7), cu, cu, 4, 4, True, 1.0, None, q)
    with pytest.raises(ValueError):
        fp8t.attn_fwd_fp8(u8(4, 8, 2).transpose(1, 2), k, k, cu, cu, 4, 4, True, 1.0, None, q)
    with pytest.raises(ValueError):
        fp8t.attn_fwd_fp8(q, k, k, cu.int(), cu, 4, 4, True, 1.0, None, q)
    with pytest.raises(TypeError):
        fp8t.rotary_embed(q.double(), i64(4), torch.zeros(2, dtype=torch.float64), q)
    with pytest.raises(ValueError):
        fp8t.rotary_embed(q, i64(3), torch.zeros(2, dtype=torch.float64), q)
    with pytest.raises(TypeError):
        fp8t.fp16_dequantize(q, torch.zeros(64, dtype=torch.float32))
    with pytest.raises(TypeError):
        fp8t.distill_loss(u8(2, 9), i64(2, 3), torch.zeros(2, 3), None, 1.0, 1.0, None, None)
    with pytest.raises(ValueError):
        fp8t.distill_loss(torch.zeros(2, 9), i64(2, 3), torch.zeros(2, 4), None, 1.0, 1.0, None, None)
